// 32 x 32 MFMA tiles of ragged attention: rows of D elements in LDS, the two ways in which they enter a product, and how tiles
// come from and go to memory.  A tile's products run on v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32; lane l = 32 h + r
// holds column r of the result and its rows 8 g + 4 h + e in element 4 g + e.
#pragma once

#include "common.h"

namespace aed {

typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();  // the score of a key that is not seen

template <typename T> struct Chunk;  // 16 bytes of a row
template <> struct Chunk<bf16_t> { typedef bf16x8 type; };
template <> struct Chunk<float> { typedef f32x4 type; };

// Rows in LDS.  The 16-byte chunks of a row change places by the row's last three bits so that (a) eight rows' chunks of one
// column, which a row operand's read touches together, lie in all banks, and (b) two neighbouring chunks of four rows, which a
// transposing read's 16 lanes touch, do too.
template <typename T, int D> struct Rows {
    typedef typename Chunk<T>::type chunk_t;
    static constexpr int kPitch = D * (int)sizeof(T), kChunks = kPitch / 16, kSteps = kChunks / 2, kTiles = D / 32;
    // float32 rows of 128: two steps of 64 of them, keys and values, would take 128 KB and leave too little for a bias and the sums of
    // its gradient (up to 79 KB).  Steps of 32 fill 64 KB, as those of other rows do at the most, but a wavefront's own rows need twice the
    // registers: one workgroup has a compute unit's.
    static constexpr int kWide = kPitch > 256;
    static constexpr int kStep = kWide ? 32 : 64;  // rows of a step of the kernels that walk over keys or queries
    static constexpr uint64_t kAll = kWide ? 0xffffffffull : ~0ull;  // a bit for each of them
    static __device__ __forceinline__ int swap_of(int row) { return ((row & 3) << 1) | ((row >> 2) & 1); }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kPitch + ((chunk ^ swap_of(row)) << 4); }
};

__device__ __forceinline__ void mma_rows(f32x16& acc, bf16x8 a, bf16x8 b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0); }
// step of 8 columns: which of them a lane half holds does not matter as long as both operands agree
__device__ __forceinline__ void mma_rows(f32x16& acc, f32x4 a, f32x4 b) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], acc, 0, 0, 0);
}

// One lane's part of 32 rows held in registers: chunks 2 s + h of row r
template <typename T, int D> struct RowFrag {
    typename Chunk<T>::type c[Rows<T, D>::kSteps];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int s = 0; s < Rows<T, D>::kSteps; ++s) c[s] = (typename Chunk<T>::type)(0);
    }
    // from memory; p: the lane's row
    __device__ __forceinline__ void load(const char* p, bool live, int half) {
        zero();
        if (live) {
#pragma unroll
            for (int s = 0; s < Rows<T, D>::kSteps; ++s) c[s] = load_global<typename Chunk<T>::type>(p + s * 32 + half * 16);
        }
    }
};

// 32 rows of LDS on their way into products.  bfloat16: load() requests the fragments, so that they travel while the matrix cores are at
// work on the ones before; float32, whose instructions take 16 times as long over a fragment, reads them at their use.
//
// AsRows: acc[i][j] = sum over D of row i of these times row j of the rows held in registers
template <typename T, int D> struct AsRows;
template <int D> struct AsRows<bf16_t, D> {
    typedef Rows<bf16_t, D> R;
    bf16x8 c[R::kSteps];
    __device__ __forceinline__ void load(const char* rows, int first, int lane) {
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s) c[s] = *reinterpret_cast<const bf16x8*>(rows + R::at(first + (lane & 31), 2 * s + (lane >> 5)));
    }
    __device__ __forceinline__ void dot(f32x16& acc, const RowFrag<bf16_t, D>& f) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s) mma_rows(acc, c[s], f.c[s]);
    }
};
template <int D> struct AsRows<float, D> {
    typedef Rows<float, D> R;
    const char* rows;
    int row, h;
    __device__ __forceinline__ void load(const char* rows_, int first, int lane) { rows = rows_, row = first + (lane & 31), h = lane >> 5; }
    __device__ __forceinline__ void dot(f32x16& acc, const RowFrag<float, D>& f) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s) mma_rows(acc, *reinterpret_cast<const f32x4*>(rows + R::at(row, 2 * s + h)), f.c[s]);
    }
};
// AsColumns: acc[t] (columns 32 t .. + 31 of D, by the 32 columns of w) += rows^T w: w[i] is the lane's weight of row 8 g + 4 h + e,
// i = 4 g + e, which is how a product of tiles leaves it.  In bfloat16 the weights are rounded here.
template <typename T, int D> struct AsColumns;
template <int D> struct AsColumns<bf16_t, D> {
    typedef Rows<bf16_t, D> R;
    bf16x8 c[2][R::kTiles];
    __device__ __forceinline__ void load(const char* rows, int first, int lane) {
        const int i = lane & 15, sub = (lane >> 4) & 1, h = lane >> 5;
        const char* p = rows + (first + 4 * h + (i >> 2)) * R::kPitch + 8 * (i & 1);
        const int sw = ((i >> 2) << 1) | h, c0 = 2 * sub + ((i & 3) >> 1);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) {
                u32x2 v[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    v[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
                                                         p + (16 * s + 8 * u) * R::kPitch + (((4 * t + c0) ^ sw) << 4))));
                c[s][t] = __builtin_bit_cast(bf16x8, u32x4{v[0][0], v[0][1], v[1][0], v[1][1]});
            }
    }
    __device__ __forceinline__ void add(f32x16* acc, const f32x16& w) const {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = (bf16_t)w[8 * s + e];
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[s][t], b, acc[t], 0, 0, 0);
        }
    }
    // with what rounding took off the weights, too: as good as weights of 16 bits
    __device__ __forceinline__ void add_finely(f32x16* acc, const f32x16& w) const {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 b, rest;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                b[e] = (bf16_t)w[8 * s + e];
                rest[e] = (bf16_t)(w[8 * s + e] - (float)b[e]);
            }
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[s][t], b, acc[t], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[s][t], rest, acc[t], 0, 0, 0);
        }
    }
    // and that alone
    __device__ __forceinline__ void add_rest(f32x16* acc, const f32x16& w) const {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 rest;
#pragma unroll
            for (int e = 0; e < 8; ++e) rest[e] = (bf16_t)(w[8 * s + e] - (float)(bf16_t)w[8 * s + e]);
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[s][t], rest, acc[t], 0, 0, 0);
        }
    }
};
template <int D> struct AsColumns<float, D> {
    typedef Rows<float, D> R;
    const char* p;
    int r, h;
    __device__ __forceinline__ void load(const char* rows, int first, int lane) { p = rows + first * R::kPitch, r = lane & 31, h = lane >> 5; }
    __device__ __forceinline__ void add_finely(f32x16* acc, const f32x16& w) const { add(acc, w); }
    __device__ __forceinline__ void add(f32x16* acc, const f32x16& w) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = 8 * (i >> 2) + 4 * h + (i & 3), sw = ((i & 3) << 1) | h;
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t) {
                const float v = *reinterpret_cast<const float*>(p + row * R::kPitch + (((8 * t + (r >> 2)) ^ sw) << 4) + 4 * (r & 3));
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w[i], acc[t], 0, 0, 0);
            }
        }
    }
};

// N rows on their way from memory to LDS through the registers of a wavefront.  Rows that are not there are beyond the end of the
// descriptor, rows that are not seen are sent there: both come as zeros, whatever stands in their place.
template <typename T, int D, int N> struct RowStage {
    typedef Rows<T, D> R;
    static constexpr int kEach = N * R::kChunks / 64, kApart = 64 / R::kChunks;
    static_assert(N * R::kChunks % 64 == 0 && 64 % R::kChunks == 0, "a lane keeps its column");
    typename R::chunk_t c[kEach];
    // first: the first of `count` >= 1 rows; seen: bit n = row n is
    __device__ __forceinline__ void load(const char* first, int pitch, int count, uint64_t seen, int lane) {
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, (min(count, N) - 1) * pitch + R::kPitch, 0x20000);
        const int row = lane / R::kChunks, off = row * pitch + (lane % R::kChunks) * 16;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = (seen >> (row + i * kApart)) & 1 ? off : kBeyond;
            c[i] = __builtin_bit_cast(typename R::chunk_t, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, i * kApart * pitch, 0));
        }
    }
    __device__ __forceinline__ void store(char* lds, int lane) const {
        const int row = lane / R::kChunks, chunk = lane % R::kChunks;
#pragma unroll
        for (int i = 0; i < kEach; ++i) *reinterpret_cast<typename R::chunk_t*>(lds + R::at(row + i * kApart, chunk)) = c[i];
    }
    static constexpr int kBeyond = 0x40000000;  // past any descriptor's end: a step's rows span less (kAttnMaxPitch)
};
// One request: every lane's 16 bytes at base + off go to LDS byte (lds_base + 16 * lane).  base and lds_base are wavefront-uniform.  The
// compiler does not see the data arrive: loads_done_barrier() waits for it.
__device__ __forceinline__ void load_to_lds16(const char* base, int off, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n" ::"s"(lds_base), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds16(const char* p, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n" ::"s"(lds_base), "v"(p) : "memory");
}
// This wavefront's loads have arrived and its LDS accesses are done, then the barrier.  The wait is the builtin: the compiler, which keeps
// count of its own loads, knows that none is left, and does not wait for them (and with them for requests to LDS) in the loop that follows.
__device__ __forceinline__ void loads_done_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt 0, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// N rows from memory to LDS, no registers in between, by the four wavefronts of a workgroup.  A request fills 1 KB of consecutive LDS, so
// what changes places are the chunks that the lanes ask for.  Rows past `count` get the last one that is there.
template <typename T, int D, int N> struct RowFeed {
    typedef Rows<T, D> R;
    static constexpr int W = 4;
    static constexpr int kAtOnce = 64 / R::kChunks, kEach = N / (W * kAtOnce);  // rows of a request, requests of a wavefront
    static_assert(W * kAtOnce % 8 == 0 && N % (W * kAtOnce) == 0, "a lane's rows agree in what its chunk is");
    int row, chunk;
    unsigned lds0;
    __device__ __forceinline__ RowFeed(const char* lds, int wave, int lane) {
        row = wave * kAtOnce + lane / R::kChunks;
        chunk = ((lane % R::kChunks) ^ R::swap_of(row)) * 16;
        lds0 = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)lds + wave * 1024;
    }
    // the i-th of a wavefront's kEach requests
    __device__ __forceinline__ void one(int i, const char* first, int pitch, int count, int lds_offset) const {
        load_to_lds16(first, min(row + i * W * kAtOnce, count - 1) * pitch + chunk, lds0 + lds_offset + i * W * 1024);
    }
    // rows whose bit is not set come from `zeros` (kPitch bytes): what stands in their place may be infinite
    __device__ __forceinline__ void load_seen(const char* first, int pitch, uint64_t seen, const char* zeros, int lds_offset) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int n = row + i * W * kAtOnce;
            load_to_lds16(((seen >> n) & 1 ? first + (int64_t)n * pitch : zeros) + chunk, lds0 + lds_offset + i * W * 1024);
        }
    }
    __device__ __forceinline__ void load(const char* first, int pitch, int count, int lds_offset) const {
        if (count >= N) {
            const int off = row * pitch + chunk;
#pragma unroll
            for (int i = 0; i < kEach; ++i) load_to_lds16(first + (int64_t)i * (W * kAtOnce) * pitch, off, lds0 + lds_offset + i * W * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) load_to_lds16(first, min(row + i * W * kAtOnce, count - 1) * pitch + chunk, lds0 + lds_offset + i * W * 1024);
        }
    }
};

__device__ __forceinline__ void put4(char* p, f32x4 v, const float*) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void put4(char* p, f32x4 v, const bf16_t*) { store4(reinterpret_cast<bf16_t*>(p), v); }

// A wavefront's 32 result rows (row = the lane's column r, D columns in acc) to memory by way of 32 rows of its own in LDS, so that
// whole rows are written: row n goes to out + n * pitch, n < count.  scale: the lane's factor.
template <typename T, int D>
__device__ __forceinline__ void store_tile(const f32x16* acc, float scale, char* scratch, char* out, int64_t pitch, int count, int lane) {
    typedef Rows<T, D> R;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 v = {acc[t][4 * g] * scale, acc[t][4 * g + 1] * scale, acc[t][4 * g + 2] * scale, acc[t][4 * g + 3] * scale};
            const int byte = (32 * t + 8 * g + 4 * h) * (int)sizeof(T);
            put4(scratch + R::at(r, byte >> 4) + (byte & 15), v, (const T*)nullptr);
        }
    other_lanes_wrote();
    constexpr int kRowsAtOnce = 64 / R::kChunks;
    static_assert(R::kChunks <= 64, "a row is written by one instruction");
    const int row0 = lane / R::kChunks, chunk = lane % R::kChunks;
#pragma unroll
    for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
        const int n = row0 + i * kRowsAtOnce;
        const typename R::chunk_t v = *reinterpret_cast<const typename R::chunk_t*>(scratch + R::at(n, chunk));
        if (n < count) *reinterpret_cast<typename R::chunk_t*>(out + n * pitch + chunk * 16) = v;
    }
    other_lanes_wrote();
}

}  // namespace aed
