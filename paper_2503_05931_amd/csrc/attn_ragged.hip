// Attention of ragged batches, forward and backward: many rows a sequence against keys of another number, with an optional
// causal mask, byte mask of the keys and learned bias by the bucket of the distance.
//
//   s_ij = scale q_i . k_j + w[bucket(i, j)]   p = softmax of the visible   o_i = sum p v   lse_i = log sum exp s
//   dP = dO . V   delta_i = dO_i . O_i   dS = P (dP - delta)   dQ = scale dS K   dK = scale dS^T Q   dV = P^T dO
//   dw[b] = sum of dS over the pairs of bucket b
//
// Exponentials are powers of two: scores and bias carry log2 e.  Scores, softmax and sums are float32; in bfloat16 the weights
// P and dS are rounded once, where they become an operand of the second product.  No result depends on timing: whatever
// is added up has one order, and there are no atomics between wavefronts.
#include "attn_ragged.h"
#include "attn_tile.h"
#include "device_once.h"

namespace aed {

namespace {

constexpr int kKeys = 64;  // keys of a step of the tiled kernels

__device__ __forceinline__ float max_halves(float v) {
    const u32x2 a = swap32(v);
    return fmaxf(bits_f32(a[0]), bits_f32(a[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const u32x2 a = swap32(v);
    return bits_f32(a[0]) + bits_f32(a[1]);
}
__device__ __forceinline__ float base_of(float m) { return m == kNone ? 0.f : m; }

// which of the 64 keys from `first` on are there and seen, one bit each
__device__ __forceinline__ uint64_t seen_keys(const RaggedArgs& a, int64_t k_row, int first, int end, int lane) {
    const int key = first + lane;
    bool ok = key < end;
    if (a.key_mask && ok) ok = load_global<uint8_t>(a.key_mask + k_row + key) != 0;
    return __ballot(ok);
}
// and by a query row at place `pos`
__device__ __forceinline__ uint64_t seen_from(uint64_t seen, int first, int pos, int causal) {
    if (!causal) return seen;
    const int last = pos - first;  // the last one that it sees
    return last >= 63 ? seen : last < 0 ? 0 : seen & ((2ull << last) - 1);
}

// ---- bias: in LDS by key - query + max_distance, both ends standing for all beyond ----
template <typename T> __device__ __forceinline__ void bias_to_lds(const RaggedArgs& a, float* w, int head) {
    for (int i = threadIdx.x; i < a.span; i += blockDim.x)
        w[i] = kLog2e * to_f32(load_global<T>(static_cast<const T*>(a.bias) + (int64_t)a.bucket_of[i] * a.heads + head));
}
enum { kInside, kAllFar, kAllNear, kMixed };
// Where the distances of a tile of 32 keys from `key` on and 32 queries from `pos` on lie.  at: place of the first of either
__device__ __forceinline__ int bias_region(const RaggedArgs& a, int key, int pos, int& at) {
    at = key - pos + a.max_distance;
    if (at + 31 <= 0) return kAllFar;
    if (at - 31 >= a.span - 1) return kAllNear;
    return at - 31 >= 0 && at + 31 <= a.span - 1 ? kInside : kMixed;
}
// s += bias; STEP 1: the lane is a query (its number r), elements are keys; -1: the other way about
template <int STEP> __device__ __forceinline__ void add_bias(float* s, const RaggedArgs& a, const float* w, int key, int pos, int r, int h) {
    int at;
    const int region = bias_region(a, key, pos, at);
    if (region == kAllFar || region == kAllNear) {
        const float b = w[region == kAllFar ? 0 : a.span - 1];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += b;
        return;
    }
    at += STEP * (4 * h - r);
    if (region == kInside) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += w[at + STEP * (8 * (i >> 2) + (i & 3))];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += w[min(max(at + STEP * (8 * (i >> 2) + (i & 3)), 0), a.span - 1)];
    }
}
// Adds the gradients of a tile (lane = query) to sums by distance.  mine: this lane half's own sums, so that no two lanes of an
// instruction meet and every sum has one order; far, near: what lies at and beyond the ends, kept by lane.
__device__ __forceinline__ void add_distances(const float* ds, const RaggedArgs& a, float* mine, float& far, float& near, int key, int pos, int r, int h) {
    int at;
    const int region = bias_region(a, key, pos, at);
    if (region == kAllFar || region == kAllNear) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += ds[i];
        if (region == kAllFar) far += sum;
        else near += sum;
        return;
    }
    at += 4 * h - r;
    if (region == kInside) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            __hip_atomic_fetch_add(mine + at + 8 * (i >> 2) + (i & 3), ds[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int n = at + 8 * (i >> 2) + (i & 3);
            if (n <= 0) far += ds[i];
            else if (n >= a.span - 1) near += ds[i];
            else __hip_atomic_fetch_add(mine + n, ds[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    }
}

// scores of a tile (lane = query): scaled, biased, those of keys that are not seen (bits of `seen`) out of the way
template <bool BIAS>
__device__ __forceinline__ void finish_scores(float* s, const f32x16& acc, const RaggedArgs& a, float scale2, const float* w, uint32_t seen, int key, int pos, int r, int h) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = acc[i] * scale2;
    if constexpr (BIAS) add_bias<1>(s, a, w, key, pos, r, h);
    if (__ballot(seen != 0xffffffffu) != 0) {
        const uint32_t mine = seen >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (mine >> (8 * (i >> 2) + (i & 3))) & 1 ? s[i] : kNone;
    }
}

// Softmax of a lane's row in passing: maximum so far, and the lane half's share of the sum
struct Running {
    float m = kNone, l = 0.f;
    template <int TILES> __device__ __forceinline__ void scale_to(float m_tile, f32x16* acc, float& base) {
        const float m_new = fmaxf(m, m_tile);
        base = base_of(m_new);
        if (__ballot(m_new > m) != 0) {
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            l *= alpha;
#pragma unroll
            for (int t = 0; t < TILES; ++t) acc[t] *= alpha;
            m = m_new;
        }
    }
};
// one tile of scores to weights; the sum goes to l
__device__ __forceinline__ void to_weights(float* s, float base, float& l) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(s[i] - base);
        l += s[i];
    }
}
__device__ __forceinline__ float max_of(const float* s) {
    float m = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
    return m;
}

template <int TILES> __device__ __forceinline__ void clear(f32x16* acc) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
}

}  // namespace

// ---------------------------------------------------------------- forward, many rows
// A workgroup takes 128 query rows of a head, 32 a wavefront, and walks the keys 64 at a time: two buffers in LDS, the next step's keys and
// values on their way in registers meanwhile.
template <typename T, int D, bool BIAS> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_forward_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kBuf = 2 * kKeys * R::kPitch;
    float* const w = reinterpret_cast<float*>(lds + 2 * kBuf);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const RaggedItem it = a.items[blockIdx.x / a.heads];
    const int head = blockIdx.x % a.heads, row0 = it.q_row + 32 * wave, count = min(max(it.rows - 32 * wave, 0), 32), pos = it.pos + 32 * wave;
    const int64_t k_head = (int64_t)(head / a.share) * a.k.head, v_head = (int64_t)(head / a.share) * a.v.head;
    const char* const kp = a.k.p + it.k_row * a.k.row + k_head;
    const char* const vp = a.v.p + it.k_row * a.v.row + v_head;
    if constexpr (BIAS) bias_to_lds<T>(a, w, head);
    RowFrag<T, D> q;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, r < count, h);
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    Running run;
    const float scale2 = a.scale * kLog2e;
    RowStage<T, D, kKeys, 256> ks, vs;
    uint64_t seen = 0;
    if (it.k_begin < it.k_end) {
        seen = seen_keys(a, it.k_row, it.k_begin, it.k_end, lane);
        ks.load(kp + it.k_begin * a.k.row, a.k.row, seen, tid);
        vs.load(vp + it.k_begin * a.v.row, a.v.row, seen, tid);
        ks.store(lds, tid);
        vs.store(lds + kBuf / 2, tid);
    }
    lds_barrier();
    int buf = 0;
    for (int k0 = it.k_begin; k0 < it.k_end; k0 += kKeys) {
        const bool more = k0 + kKeys < it.k_end;
        uint64_t seen_next = 0;
        if (more) {
            seen_next = seen_keys(a, it.k_row, k0 + kKeys, it.k_end, lane);
            ks.load(kp + (k0 + kKeys) * a.k.row, a.k.row, seen_next, tid);
            vs.load(vp + (k0 + kKeys) * a.v.row, a.v.row, seen_next, tid);
        }
        const char* const kb = lds + buf * kBuf;
        const char* const vb = kb + kBuf / 2;
        const uint64_t mine = seen_from(seen, k0, pos + r, a.causal);
        if (__ballot(mine != 0) != 0 && count > 0) {
            float s[2][16];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                finish_scores<BIAS>(s[u], dot_rows<T, D>(kb, 32 * u, q, lane), a, scale2, w, (uint32_t)(mine >> (32 * u)), k0 + 32 * u, pos, r, h);
            float base;
            run.scale_to<R::kTiles>(max_halves(fmaxf(max_of(s[0]), max_of(s[1]))), acc, base);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                to_weights(s[u], base, run.l);
                add_weighted<D>(acc, vb, 32 * u, s[u], lane, (const T*)nullptr);
            }
        }
        if (more) {
            ks.store(lds + (buf ^ 1) * kBuf, tid);
            vs.store(lds + (buf ^ 1) * kBuf + kBuf / 2, tid);
        }
        lds_barrier();
        seen = seen_next;
        buf ^= 1;
    }
    const float l = sum_halves(run.l);
    if (it.part < 0) {
        store_tile<T, D>(acc, l > 0.f ? 1.f / l : l, lds + wave * 32 * R::kPitch, a.o.p + (int64_t)row0 * a.o.row + head * a.o.head, a.o.row, count, lane);
        if (h == 0 && r < count) a.lse[(int64_t)(row0 + r) * a.heads + head] = kLn2 * (run.m + __builtin_amdgcn_logf(l));
    } else if (r < count) {
        const int64_t at = ((int64_t)it.part * a.heads + head) * kAttnRows + 32 * wave + r;
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                store4(a.part_o + at * D + 32 * t + 8 * g + 4 * h, f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]});
        if (h == 0) a.part_ml[at] = float2{run.m, l};
    }
}

// ---------------------------------------------------------------- forward, few rows
// A workgroup takes up to 32 query rows of a head; its four wavefronts take 32 keys each in turn, through rows of LDS of their own, and
// join their sums at the end.  The matrix cores are mostly idle here: what counts is that keys and values stream.
template <typename T, int D, bool BIAS> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_few_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kMine = 2 * 32 * R::kPitch;
    float* const w = reinterpret_cast<float*>(lds + 4 * kMine);
    __shared__ float2 ml[4][32];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const RaggedItem it = a.items[blockIdx.x / a.heads];
    const int head = blockIdx.x % a.heads, row0 = it.q_row, count = it.rows, pos = it.pos;
    const int64_t k_head = (int64_t)(head / a.share) * a.k.head, v_head = (int64_t)(head / a.share) * a.v.head;
    const char* const kp = a.k.p + it.k_row * a.k.row + k_head;
    const char* const vp = a.v.p + it.k_row * a.v.row + v_head;
    char* const kb = lds + wave * kMine;
    char* const vb = kb + kMine / 2;
    RowStage<T, D, 32, 64> ks, vs;
    uint64_t seen = 0;
    int k0 = it.k_begin + 32 * wave;
    if (k0 < it.k_end) {
        seen = seen_keys(a, it.k_row, k0, it.k_end, lane);
        ks.load(kp + k0 * a.k.row, a.k.row, seen, lane);
        vs.load(vp + k0 * a.v.row, a.v.row, seen, lane);
    }
    RowFrag<T, D> q;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, r < count, h);
    if constexpr (BIAS) {
        bias_to_lds<T>(a, w, head);
        lds_barrier();
    }
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    Running run;
    const float scale2 = a.scale * kLog2e;
    for (; k0 < it.k_end; k0 += 128) {
        ks.store(kb, lane);
        vs.store(vb, lane);
        other_lanes_wrote();
        const uint32_t mine = (uint32_t)seen_from(seen, k0, pos + r, a.causal);
        if (k0 + 128 < it.k_end) {
            seen = seen_keys(a, it.k_row, k0 + 128, it.k_end, lane);
            ks.load(kp + (k0 + 128) * a.k.row, a.k.row, seen, lane);
            vs.load(vp + (k0 + 128) * a.v.row, a.v.row, seen, lane);
        }
        float s[16], base;
        finish_scores<BIAS>(s, dot_rows<T, D>(kb, 0, q, lane), a, scale2, w, mine, k0, pos, r, h);
        run.scale_to<R::kTiles>(max_halves(max_of(s)), acc, base);
        to_weights(s, base, run.l);
        add_weighted<D>(acc, vb, 0, s, lane, (const T*)nullptr);
        other_lanes_wrote();
    }
    // join: maximum, then the sums scaled to it
    float l = sum_halves(run.l);
    if (h == 0) ml[wave][r] = float2{run.m, l};
    __syncthreads();
    float m = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, ml[i][r].x);
    const float alpha = __builtin_amdgcn_exp2f(run.m - base_of(m));
    float* const sums = reinterpret_cast<float*>(lds);  // [4][count][D]; the wavefronts' rows are done with
    if (r < count) {
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(sums + (wave * count + r) * D + 32 * t + 8 * g + 4 * h) =
                    f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]} * alpha;
    }
    __syncthreads();
    for (int i = tid; i < count * (D / 4); i += 256) {
        const int row = i / (D / 4), c = i % (D / 4) * 4;
        float top = kNone, total = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, ml[j][row].x);
#pragma unroll
        for (int j = 0; j < 4; ++j) total += ml[j][row].y * __builtin_amdgcn_exp2f(ml[j][row].x - base_of(top));
        f32x4 v = *reinterpret_cast<const f32x4*>(sums + row * D + c);
#pragma unroll
        for (int j = 1; j < 4; ++j) v += *reinterpret_cast<const f32x4*>(sums + (j * count + row) * D + c);
        if (it.part < 0) {
            v *= total > 0.f ? 1.f / total : total;
            put4(a.o.p + (int64_t)(row0 + row) * a.o.row + head * a.o.head + c * sizeof(T), v, (const T*)nullptr);
            if (c == 0) a.lse[(int64_t)(row0 + row) * a.heads + head] = kLn2 * (top + __builtin_amdgcn_logf(total));
        } else {
            const int64_t at = ((int64_t)it.part * a.heads + head) * kAttnFew + row;
            store4(a.part_o + at * D + c, v);
            if (c == 0) a.part_ml[at] = float2{top, total};
        }
    }
}

// ---------------------------------------------------------------- parts of rows whose keys were split
template <typename T, int D> __global__ __launch_bounds__(256) void attn_join_kernel(RaggedArgs a, int tile_rows) {
    const RaggedJoin j = a.joins[blockIdx.x];
    const int head = blockIdx.y, per = D / 4, at = blockIdx.z * 256 + threadIdx.x;
    if (at >= j.rows * per) return;
    const int row = at / per, c = at % per * 4;
    const int64_t first = ((int64_t)j.part * a.heads + head) * tile_rows + row, step = (int64_t)a.heads * tile_rows;
    float m = kNone;
    for (int i = 0; i < j.n_parts; ++i) m = fmaxf(m, a.part_ml[first + i * step].x);
    float l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < j.n_parts; ++i) {
        const float2 p = a.part_ml[first + i * step];
        const float alpha = __builtin_amdgcn_exp2f(p.x - base_of(m));
        l += p.y * alpha;
        v += load4(a.part_o + (first + i * step) * D + c) * alpha;
    }
    v *= l > 0.f ? 1.f / l : l;
    put4(a.o.p + (int64_t)(j.q_row + row) * a.o.row + head * a.o.head + c * sizeof(T), v, (const T*)nullptr);
    if (c == 0) a.lse[(int64_t)(j.q_row + row) * a.heads + head] = kLn2 * (m + __builtin_amdgcn_logf(l));
}

// ---------------------------------------------------------------- query gradients, delta, and the bias's
// The forward kernel's walk with two products to a tile of scores (K Q^T and V dO^T, transposed, a lane being a query) and one
// more for dQ.  delta is left for the key gradients' kernel, without the error that the rounded output leaves in it: a row's dS add up
// to 0, so what they do add up to is what delta lacks.
template <typename T, int D, bool BIAS> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_dq_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kBuf = 2 * kKeys * R::kPitch;
    float* const w = reinterpret_cast<float*>(lds + kBuf);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    float* const sums = w + a.span;  // [wavefront, half][span]
    const int item = blockIdx.x / a.heads;
    const RaggedItem it = a.items[item];
    const int head = blockIdx.x % a.heads, row0 = it.q_row + 32 * wave, count = min(max(it.rows - 32 * wave, 0), 32), pos = it.pos + 32 * wave;
    const int64_t k_head = (int64_t)(head / a.share) * a.k.head, v_head = (int64_t)(head / a.share) * a.v.head;
    const char* const kp = a.k.p + it.k_row * a.k.row + k_head;
    const char* const vp = a.v.p + it.k_row * a.v.row + v_head;
    if constexpr (BIAS) {
        bias_to_lds<T>(a, w, head);
        for (int i = tid; i < 8 * a.span; i += 256) sums[i] = 0.f;
    }
    RowFrag<T, D> q, d_o;
    const bool live = r < count;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, live, h);
    d_o.load(a.d_o.p + (int64_t)(row0 + r) * a.d_o.row + head * a.d_o.head, live, h);
    float delta = 0.f, lse2 = kNone;
    {
        RowFrag<T, D> o;
        o.load(a.o.p + (int64_t)(row0 + r) * a.o.row + head * a.o.head, live, h);
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 16 / (int)sizeof(T); ++e) delta += to_f32((T)o.c[s][e]) * to_f32((T)d_o.c[s][e]);
        delta = sum_halves(delta);
        if (live) lse2 = kLog2e * a.lse[(int64_t)(row0 + r) * a.heads + head];
    }
    // a row that sees nothing has lse -inf, and none of its keys' bits are set: its weights become 0 by way of the scores
    const float base = base_of(lse2), scale2 = a.scale * kLog2e;
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    float far = 0.f, near = 0.f, rest = 0.f;
    RowStage<T, D, kKeys, 256> ks, vs;
    uint64_t seen = 0;
    if (it.k_begin < it.k_end) {
        seen = seen_keys(a, it.k_row, it.k_begin, it.k_end, lane);
        ks.load(kp + it.k_begin * a.k.row, a.k.row, seen, tid);
        vs.load(vp + it.k_begin * a.v.row, a.v.row, seen, tid);
    }
    for (int k0 = it.k_begin; k0 < it.k_end; k0 += kKeys) {
        ks.store(lds, tid);
        vs.store(lds + kBuf / 2, tid);
        lds_barrier();
        const uint64_t mine = live ? seen_from(seen, k0, pos + r, a.causal) : 0;
        if (k0 + kKeys < it.k_end) {
            seen = seen_keys(a, it.k_row, k0 + kKeys, it.k_end, lane);
            ks.load(kp + (k0 + kKeys) * a.k.row, a.k.row, seen, tid);
            vs.load(vp + (k0 + kKeys) * a.v.row, a.v.row, seen, tid);
        }
        if (__ballot(mine != 0) != 0) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float s[16];
                finish_scores<BIAS>(s, dot_rows<T, D>(lds, 32 * u, q, lane), a, scale2, w, (uint32_t)(mine >> (32 * u)), k0 + 32 * u, pos, r, h);
                const f32x16 dp = dot_rows<T, D>(lds + kBuf / 2, 32 * u, d_o, lane);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[i] = __builtin_amdgcn_exp2f(s[i] - base) * (dp[i] - delta);
                    rest += s[i];
                }
                if constexpr (BIAS) add_distances(s, a, sums + (2 * wave + h) * a.span, far, near, k0 + 32 * u, pos, r, h);
                add_weighted<D>(acc, lds, 32 * u, s, lane, (const T*)nullptr);
            }
        }
        lds_barrier();
    }
    rest = sum_halves(rest);
    if (live && h == 0) a.delta[(int64_t)(row0 + r) * a.heads + head] = delta + rest;
    lds_barrier();
    store_tile<T, D>(acc, a.scale, lds + wave * 32 * R::kPitch, a.dq.p + (int64_t)row0 * a.dq.row + head * a.dq.head, a.dq.row, count, lane);
    if constexpr (BIAS) {
        // the ends' sums by wavefront, then the eight sums of a distance, then a bucket's distances, which lie side by side
        far = wave_sum(far);
        near = wave_sum(near);
        lds_barrier();
        if (lane == 0) {
            sums[2 * wave * a.span] += far;
            sums[2 * wave * a.span + a.span - 1] += near;
        }
        lds_barrier();
        for (int i = tid; i < a.span; i += 256) {
            float v = 0.f;
            for (int j = 0; j < 8; ++j) v += sums[j * a.span + i];
            w[i] = v;
        }
        lds_barrier();
        float* const out = a.part_bias + ((int64_t)item * a.heads + head) * a.buckets;
        for (int b = tid; b < a.buckets; b += 256) {
            float v = 0.f;
            for (int i = a.bucket_range[b].x; i < a.bucket_range[b].y; ++i) v += w[i];
            out[b] = v;
        }
    }
}

// ---------------------------------------------------------------- key and value gradients
// A workgroup takes 128 keys of a key head, 32 a wavefront (a lane being a key), and walks the query rows of all heads that share it.
template <typename T, int D, bool BIAS> __global__ __launch_bounds__(256, 1) void attn_dkv_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    constexpr int kRows = 64;
    extern __shared__ __align__(16) char lds[];
    constexpr int kBuf = 2 * kRows * R::kPitch;
    float* const row_lse = reinterpret_cast<float*>(lds + kBuf);  // [kRows], then [kRows] of delta
    float* const row_delta = row_lse + kRows;
    float* const w = row_delta + kRows;
    const int kv_heads = a.heads / a.share;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const RaggedItem it = a.items[blockIdx.x / kv_heads];
    const int kv_head = blockIdx.x % kv_heads, count = min(max(it.rows - 32 * wave, 0), 32), key0 = it.pos + 32 * wave;
    const int64_t k_row0 = it.k_row + 32 * wave;
    bool live = r < count;
    if (a.key_mask && live) live = load_global<uint8_t>(a.key_mask + k_row0 + r) != 0;
    RowFrag<T, D> k, v;
    k.load(a.k.p + (k_row0 + r) * a.k.row + kv_head * a.k.head, live, h);
    v.load(a.v.p + (k_row0 + r) * a.v.row + kv_head * a.v.head, live, h);
    f32x16 dk[R::kTiles], dv[R::kTiles];
    clear<R::kTiles>(dk);
    clear<R::kTiles>(dv);
    const float scale2 = a.scale * kLog2e;
    for (int head = kv_head * a.share; head < (kv_head + 1) * a.share; ++head) {
        if constexpr (BIAS) {
            lds_barrier();
            bias_to_lds<T>(a, w, head);
        }
        const char* const qp = a.q.p + (int64_t)it.q_row * a.q.row + head * a.q.head;
        const char* const gp = a.d_o.p + (int64_t)it.q_row * a.d_o.row + head * a.d_o.head;
        RowStage<T, D, kRows, 256> qs, gs;
        float stat = 0.f;
        auto fetch = [&](int q0) {
            const int n = it.k_end - q0;
            const uint64_t there = n >= 64 ? ~0ull : (1ull << n) - 1;
            qs.load(qp + q0 * a.q.row, a.q.row, there, tid);
            gs.load(gp + q0 * a.d_o.row, a.d_o.row, there, tid);
            if (tid < 2 * kRows) {  // a row that is not there or sees nothing: its weights are 2^-inf
                const int row = tid & (kRows - 1);
                stat = tid < kRows ? -kNone : 0.f;
                if (row < n) {
                    const int64_t at = (int64_t)(it.q_row + q0 + row) * a.heads + head;
                    stat = tid < kRows ? kLog2e * a.lse[at] : a.delta[at];
                    if (stat == kNone) stat = -kNone;
                }
            }
        };
        if (it.k_begin < it.k_end) fetch(it.k_begin);
        for (int q0 = it.k_begin; q0 < it.k_end; q0 += kRows) {
            qs.store(lds, tid);
            gs.store(lds + kBuf / 2, tid);
            if (tid < 2 * kRows) row_lse[tid] = stat;
            lds_barrier();
            const int rows = it.k_end - q0;
            if (q0 + kRows < it.k_end) fetch(q0 + kRows);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int first = q0 + 32 * u;
                // key0 counts in query rows: row i sees the keys up to its own place
                if (32 * u >= rows || count == 0 || (a.causal && first + 31 < key0)) continue;
                const f32x16 x = dot_rows<T, D>(lds, 32 * u, k, lane);
                float p[16], ds[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = x[i] * scale2;
                if constexpr (BIAS) add_bias<-1>(p, a, w, key0, first, r, h);
                const f32x16 dp = dot_rows<T, D>(lds + kBuf / 2, 32 * u, v, lane);
                const int last = a.causal ? key0 + r - first - 4 * h : -4;  // rows before that one do not see the key
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 lse = *reinterpret_cast<const f32x4*>(row_lse + 32 * u + 8 * g + 4 * h);
                    const f32x4 delta = *reinterpret_cast<const f32x4*>(row_delta + 32 * u + 8 * g + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * g + e;
                        p[i] = live && 8 * g + e >= last ? __builtin_amdgcn_exp2f(p[i] - lse[e]) : 0.f;
                        ds[i] = p[i] * (dp[i] - delta[e]);
                    }
                }
                add_weighted<D>(dv, lds + kBuf / 2, 32 * u, p, lane, (const T*)nullptr);
                add_weighted<D>(dk, lds, 32 * u, ds, lane, (const T*)nullptr);
            }
            lds_barrier();
        }
    }
    lds_barrier();
    char* const scratch = lds + wave * 32 * R::kPitch;
    store_tile<T, D>(dk, a.scale, scratch, a.dk.p + k_row0 * a.dk.row + kv_head * a.dk.head, a.dk.row, count, lane);
    store_tile<T, D>(dv, 1.f, scratch, a.dv.p + k_row0 * a.dv.row + kv_head * a.dv.head, a.dv.row, count, lane);
}

// ---------------------------------------------------------------- bias gradient: the items' sums of one bucket and head
template <typename T> __global__ __launch_bounds__(64) void attn_dbias_kernel(RaggedArgs a, int items, T* d_bias) {
    const int b = blockIdx.x, head = blockIdx.y;
    float v = 0.f;
    for (int i = threadIdx.x; i < items; i += 64) v += a.part_bias[((int64_t)i * a.heads + head) * a.buckets + b];
    v = wave_sum(v);
    if (threadIdx.x == 0) d_bias[(int64_t)b * a.heads + head] = from_f32<T>(v);
}

// ---------------------------------------------------------------- launches
namespace {

template <typename K> hipError_t launch(K kernel, DeviceOnce& once, int64_t blocks, size_t lds, const RaggedArgs& a, hipStream_t s) {
    hipError_t e = once.run([&] { return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - 1024); });
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)blocks), dim3(256), lds, s>>>(a);
    return hipGetLastError();
}
// f(type, head size, bias)
template <typename F> hipError_t by_kind(int head_dim, bool bf16, bool bias, F f) {
    if (bf16) {
        if (head_dim == 128) return bias ? f((bf16_t*)nullptr, std::integral_constant<int, 128>(), std::true_type()) : f((bf16_t*)nullptr, std::integral_constant<int, 128>(), std::false_type());
        return bias ? f((bf16_t*)nullptr, std::integral_constant<int, 64>(), std::true_type()) : f((bf16_t*)nullptr, std::integral_constant<int, 64>(), std::false_type());
    }
    if (head_dim == 128) return bias ? f((float*)nullptr, std::integral_constant<int, 128>(), std::true_type()) : f((float*)nullptr, std::integral_constant<int, 128>(), std::false_type());
    return bias ? f((float*)nullptr, std::integral_constant<int, 64>(), std::true_type()) : f((float*)nullptr, std::integral_constant<int, 64>(), std::false_type());
}

}  // namespace

hipError_t launch_attn_forward(const RaggedArgs& a, int head_dim, bool bf16, bool few, int items, hipStream_t s) {
    if (items == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr, [&](auto* t, auto d, auto bias) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool B = decltype(bias)::value;
        static DeviceOnce once_few, once_many;
        const size_t w = B ? a.span * sizeof(float) : 0;
        if (few) return launch(attn_few_kernel<T, D, B>, once_few, (int64_t)items * a.heads, 4 * 2 * 32 * Rows<T, D>::kPitch + w, a, s);
        return launch(attn_forward_kernel<T, D, B>, once_many, (int64_t)items * a.heads, 4 * kKeys * Rows<T, D>::kPitch + w, a, s);
    });
}

hipError_t launch_attn_join(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, int joins, hipStream_t s) {
    if (joins == 0) return hipSuccess;
    return by_kind(head_dim, bf16, false, [&](auto* t, auto d, auto) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        attn_join_kernel<T, D><<<dim3(joins, a.heads, (tile_rows * (D / 4) + 255) / 256), 256, 0, s>>>(a, tile_rows);
        return hipGetLastError();
    });
}

hipError_t launch_attn_dq(const RaggedArgs& a, int head_dim, bool bf16, int items, hipStream_t s) {
    if (items == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr, [&](auto* t, auto d, auto bias) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool B = decltype(bias)::value;
        static DeviceOnce once;
        return launch(attn_dq_kernel<T, D, B>, once, (int64_t)items * a.heads, 2 * kKeys * Rows<T, D>::kPitch + (B ? 9 * a.span * sizeof(float) : 0), a, s);
    });
}

hipError_t launch_attn_dkv(const RaggedArgs& a, int head_dim, bool bf16, int items, hipStream_t s) {
    if (items == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr, [&](auto* t, auto d, auto bias) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool B = decltype(bias)::value;
        static DeviceOnce once;
        return launch(attn_dkv_kernel<T, D, B>, once, (int64_t)items * (a.heads / a.share), 2 * 64 * Rows<T, D>::kPitch + 512 + (B ? a.span * sizeof(float) : 0), a, s);
    });
}

hipError_t launch_attn_dbias(const RaggedArgs& a, bool bf16, int items, void* d_bias, hipStream_t s) {
    const dim3 grid(a.buckets, a.heads);
    if (bf16) attn_dbias_kernel<bf16_t><<<grid, 64, 0, s>>>(a, items, static_cast<bf16_t*>(d_bias));
    else attn_dbias_kernel<float><<<grid, 64, 0, s>>>(a, items, static_cast<float*>(d_bias));
    return hipGetLastError();
}

}  // namespace aed
