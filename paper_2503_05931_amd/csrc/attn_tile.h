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
    static constexpr int kWide = kPitch > 256;  // a workgroup's rows fill the LDS of half a CU and more: one of them has all its registers
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

// acc[i][j] = sum over D of a row i in LDS (first .. first + 31 of `rows`) times row j held in registers
template <typename T, int D> __device__ __forceinline__ f32x16 dot_rows(const char* rows, int first, const RowFrag<T, D>& f, int lane) {
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < Rows<T, D>::kSteps; ++s)
        mma_rows(acc, *reinterpret_cast<const typename Chunk<T>::type*>(rows + Rows<T, D>::at(first + (lane & 31), 2 * s + (lane >> 5))), f.c[s]);
    return acc;
}

// acc[t] (columns 32 t .. + 31 of D, by the 32 columns of w) += rows^T w: w[i] is the lane's weight of LDS row first + 8 g + 4 h + e,
// i = 4 g + e, which is how a product of tiles leaves it.  In bfloat16 the weights are rounded here.
template <int D> __device__ __forceinline__ void add_weighted(f32x16* acc, const char* rows, int first, const float* w, int lane, const bf16_t*) {
    typedef Rows<bf16_t, D> R;
    const int i = lane & 15, sub = (lane >> 4) & 1, h = lane >> 5;
    const char* p = rows + (first + 4 * h + (i >> 2)) * R::kPitch + 8 * (i & 1);
    const int sw = ((i >> 2) << 1) | h, c0 = 2 * sub + ((i & 3) >> 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (bf16_t)w[8 * s + e];
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t) {
            u32x2 v[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                v[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
                                                     p + (16 * s + 8 * u) * R::kPitch + (((4 * t + c0) ^ sw) << 4))));
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{v[0][0], v[0][1], v[1][0], v[1][1]}), b, acc[t], 0, 0, 0);
        }
    }
}
template <int D> __device__ __forceinline__ void add_weighted(f32x16* acc, const char* rows, int first, const float* w, int lane, const float*) {
    typedef Rows<float, D> R;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i >> 2) + 4 * h + (i & 3), sw = ((i & 3) << 1) | h;
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t) {
            const float v = *reinterpret_cast<const float*>(rows + (first + row) * R::kPitch + (((8 * t + (r >> 2)) ^ sw) << 4) + 4 * (r & 3));
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w[i], acc[t], 0, 0, 0);
        }
    }
}

// N rows on their way from memory to LDS through the registers of THREADS threads
template <typename T, int D, int N, int THREADS> struct RowStage {
    typedef Rows<T, D> R;
    static constexpr int kEach = N * R::kChunks / THREADS;
    static_assert(N * R::kChunks % THREADS == 0 && THREADS % R::kChunks == 0, "a thread keeps its column");
    typename R::chunk_t c[kEach];
    // live: bit n = row n is there and is seen (others are zeros: what stands in their place may be infinite)
    __device__ __forceinline__ void load(const char* first, int64_t pitch, uint64_t live, int tid) {
        const int row = tid / R::kChunks;
        const char* p = first + row * pitch + (tid % R::kChunks) * 16;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int n = row + i * (THREADS / R::kChunks);
            c[i] = (typename R::chunk_t)(0);
            if ((live >> n) & 1) c[i] = load_global<typename R::chunk_t>(p + (int64_t)i * (THREADS / R::kChunks) * pitch);
        }
    }
    __device__ __forceinline__ void store(char* lds, int tid) const {
        const int row = tid / R::kChunks, chunk = tid % R::kChunks;
#pragma unroll
        for (int i = 0; i < kEach; ++i) *reinterpret_cast<typename R::chunk_t*>(lds + R::at(row + i * (THREADS / R::kChunks), chunk)) = c[i];
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
