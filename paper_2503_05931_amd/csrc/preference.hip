// The loss of paired log ratios, from the logits of both transcripts, and its gradient by them.
//
//   lp_t = z_t[y_t] - lse(z_t)   ratio_s = sum of lp_t - ref_t   x = beta (ratio of the preferred - ratio of the other)
//   loss = mean of -(1 - eps) log sigmoid(x) - eps log sigmoid(-x)   dz_t = (d loss / d ratio) (onehot(y_t) - softmax(z_t))
//
// Bound by memory: forward reads the logits once, backward reads them again and writes as much.  A row's maximum and sum are
// taken in one pass and kept apart: what is subtracted from a logit is its row's maximum, exactly, so that large logits cost no
// digits.  The sums over a sequence are of differences to the reference, which are small, and have one order.  A gradient is rounded
// once, where it is stored.
// 8 141 rows of 4 096 logits in bfloat16, 67 MB: reading them takes 13 us (5.1 TB/s), the pairs 4.8, the gradient 21.8 (133 MB, 6.1 TB/s:
// the logits are partly still in the last cache).
#include "common.h"
#include "preference.h"

#include <type_traits>

namespace aed {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T> struct Vec;
template <> struct Vec<bf16_t> { typedef bf16x8 type; static constexpr int n = 8; };
template <> struct Vec<float> { typedef f32x4 type; static constexpr int n = 4; };

__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_mov<0xB1>(v));
    v = fmaxf(v, dpp_mov<0x4E>(v));
    v = fmaxf(v, dpp_mov<0x141>(v));
    v = fmaxf(v, dpp_mov<0x140>(v));
    return rows4_max(v);
}
// A row of any alignment: `head` elements up to a 16-byte boundary, `vecs` whole vectors, then the rest
template <typename T> struct RowParts {
    int head, vecs, tail;  // tail: first element behind the vectors
    __device__ __forceinline__ RowParts(const T* p, int n) {
        head = min(n, (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T));
        vecs = (n - head) / Vec<T>::n;
        tail = head + vecs * Vec<T>::n;
    }
    // the one element outside the vectors that lane l (of 64) looks after, or -1
    __device__ __forceinline__ int loose(int lane, int n) const {
        if (lane < head) return lane;
        const int at = tail + lane - head;
        return at < n && lane >= head ? at : -1;
    }
};
__device__ __forceinline__ bool scored(int label, int vocab) { return label >= 0 && label < vocab; }

}  // namespace

namespace {

// -log sigmoid(x)
__device__ __forceinline__ float loss_of(float x) { return fmaxf(-x, 0.f) + log1pf(expf(-fabsf(x))); }

// A workgroup of W wavefronts: sixteen lanes add up a sequence, 4 W sequences at once, then the pairs' losses are added.  gain(i): of row i
template <int W, typename G> __device__ __forceinline__ void add_pairs(const PreferenceArgs& a, G gain) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = threadIdx.x & 15;
    __shared__ float part[W];
    float mine = 0.f;
    for (int s = threadIdx.x >> 4; s < 2 * a.pairs; s += 4 * W) {  // both sequences of a pair are a wavefront's
        const int first = a.seq_start[s], end = a.seq_start[s + 1];
        float v = 0.f;
#pragma unroll 8
        for (int i = first + sub; i < end; i += 16) v += gain(i);
        v = row16_sum(v);
        if (sub == 0) a.ratio[s] = v;
        const u32x2 both = swap16(v);  // of lanes l and l ^ 16: the preferred one and the other
        const float x = a.beta * (bits_f32(both[0]) - bits_f32(both[1]));
        if ((lane & 31) == 0) mine += (1.f - a.smoothing) * loss_of(x) + (a.smoothing > 0.f ? a.smoothing * loss_of(-x) : 0.f);
    }
    mine = wave_sum(mine);
    if (lane == 0) part[wave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        float v = 0.f;
        for (int i = 0; i < W; ++i) v += part[i];
        a.loss[0] = v / (float)a.pairs;
    }
}

// a lane's vectors of a row, S of them at once, into its maximum and sum
template <typename T, int S> __device__ __forceinline__ void take(const typename Vec<T>::type* zv, int vecs, int lane, float& m, float& l) {
    typedef typename Vec<T>::type V;
    constexpr int N = Vec<T>::n;
    for (int v0 = lane; v0 < vecs; v0 += 64 * S) {
        V x[S];
#pragma unroll
        for (int i = 0; i < S; ++i) x[i] = zv[min(v0 + 64 * i, vecs - 1)];
        float y[S][N], top = m;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const bool there = v0 + 64 * i < vecs;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                y[i][e] = there ? to_f32((T)x[i][e]) : -__builtin_inff();
                top = fmaxf(top, y[i][e]);
            }
        }
        const float base = top == -__builtin_inff() ? 0.f : top;
        l *= __builtin_amdgcn_exp2f((m - base) * kLog2e);
        m = top;
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) l += __builtin_amdgcn_exp2f((y[i][e] - base) * kLog2e);
    }
}

// (log-probability of the label less the reference's, maximum and log of the rest) of a row, by a wavefront; all lanes have them
struct RowResult {
    float gain = 0.f;
    float2 lse = {0.f, 0.f};
};
template <typename T, int S> __device__ __forceinline__ RowResult row_result(const PreferenceArgs& a, int row, int lane) {
    typedef typename Vec<T>::type V;
    RowResult r;
    const int label = a.labels[row];
    if (!scored(label, a.vocab)) return r;
    const T* const z = static_cast<const T*>(a.logits) + row * a.row_stride;
    const RowParts<T> part(z, a.vocab);
    const V* const zv = reinterpret_cast<const V*>(z + part.head);
    float m = -__builtin_inff(), l = 0.f;
    const int at = part.loose(lane, a.vocab);
    if (at >= 0) {
        m = to_f32(z[at]);
        l = m == -__builtin_inff() ? 0.f : 1.f;
    }
    take<T, S>(zv, part.vecs, lane, m, l);
    const float top = wave_max(m), base = top == -__builtin_inff() ? 0.f : top;
    l = wave_sum(l * __builtin_amdgcn_exp2f((m - base) * kLog2e));
    r.lse = float2{top, kLn2 * __builtin_amdgcn_logf(l)};
    r.gain = (to_f32(z[label]) - top) - r.lse.y - a.ref[row];
    return r;
}

}  // namespace

// One wavefront a row, S vectors of it at once: 5.1 TB/s.
// LAST: the workgroup that is the last to arrive adds up the pairs, which saves a launch.  Gains and the count of arrivals are exchanged by relaxed
// atomic accesses of device scope, which are made where all dies see them; a workgroup has waited for its stores before it is counted, and the last one
// reads only when it has seen the full count.  Which one that is changes no result: a sequence's rows are added in their order.
template <typename T, int S, bool LAST> __global__ __launch_bounds__(256) void preference_rows_kernel(PreferenceArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row < a.rows) {
        const RowResult r = row_result<T, S>(a, row, lane);
        if (lane == 0) {
            a.lse[row] = r.lse;
            if constexpr (LAST) __hip_atomic_store(&a.gain[row], r.gain, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            else a.gain[row] = r.gain;
        }
    }
    if constexpr (LAST) {
        __shared__ int last;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) last = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        add_pairs<4>(a, [&](int i) { return __hip_atomic_load(&a.gain[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
        if (threadIdx.x == 0) __hip_atomic_store(a.arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next call
    }
}

__global__ __launch_bounds__(1024) void preference_pairs_kernel(PreferenceArgs a) {
    add_pairs<16>(a, [&](int i) { return a.gain[i]; });
}

// One wavefront a row; row t's gradient is slope (onehot - softmax).  S vectors are read before the first is written: eight 21.8 us, one by one 22.6.
template <typename T, int S> __global__ __launch_bounds__(256) void preference_gradient_kernel(PreferenceArgs a) {
    typedef typename Vec<T>::type V;
    constexpr int N = Vec<T>::n;
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.rows) return;
    const int label = a.labels[row];
    const bool live = scored(label, a.vocab);
    const T* const z = static_cast<const T*>(a.logits) + row * a.row_stride;
    T* const d = static_cast<T*>(a.d_logits) + row * a.d_row_stride;
    float slope = 0.f, top = 0.f, log2_l = 0.f;
    if (live) {
        const int seq = a.seq_of[row], p = seq >> 1;
        const float x = a.beta * (a.ratio[2 * p] - a.ratio[2 * p + 1]);
        const float up = 1.f / (1.f + expf(-x)), down = 1.f / (1.f + expf(x));  // sigmoid of x and of -x
        slope = a.beta / (float)a.pairs * (a.smoothing * up - (1.f - a.smoothing) * down) * (a.d_loss ? a.d_loss[0] : 1.f);
        if (seq & 1) slope = -slope;
        const float2 lse = a.lse[row];
        top = lse.x;
        log2_l = kLog2e * lse.y;
    }
    auto gradient = [&](float x, int at) {
        const float p = slope * __builtin_amdgcn_exp2f(fmaf(x - top, kLog2e, -log2_l));
        return from_f32<T>(at == label ? slope - p : -p);
    };
    const RowParts<T> part(d, a.vocab);
    const int at = part.loose(lane, a.vocab);
    if (at >= 0) d[at] = live ? gradient(to_f32(z[at]), at) : from_f32<T>(0.f);
    V* const dv = reinterpret_cast<V*>(d + part.head);
    if (!live) {
        for (int v = lane; v < part.vecs; v += 64) dv[v] = (V)(0);
        return;
    }
    const bool same = ((uintptr_t)(z + part.head) & 15) == 0;  // logits and gradients lie alike to 16 bytes
    for (int v0 = lane; v0 < part.vecs; v0 += 64 * S) {
        V x[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const T* const from = z + part.head + min(v0 + 64 * i, part.vecs - 1) * N;
            if (same) x[i] = *reinterpret_cast<const V*>(from);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] = from[e];
            }
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int v = v0 + 64 * i;
            V y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = gradient(to_f32((T)x[i][e]), part.head + v * N + e);
            if (v < part.vecs) dv[v] = y;
        }
    }
}

namespace {

// f(type, vectors of a row that a lane holds at once).  As many as rows have, up to eight: with eight always, rows of 512 logits in bfloat16 (one vector
// a lane) take 19.5 instead of 12.4 us forward and 8.7 instead of 7.3 backward (12 800 rows), rows of 1500 (three) 20.6 instead of 16.5 forward.
template <typename F> void by_row(const PreferenceArgs& a, bool bf16, F f) {
    auto with = [&](auto* t) {
        const int vecs = a.vocab / Vec<std::remove_pointer_t<decltype(t)>>::n;
        if (vecs <= 64) f(t, std::integral_constant<int, 1>());
        else if (vecs <= 192) f(t, std::integral_constant<int, 3>());
        else f(t, std::integral_constant<int, 8>());
    };
    if (bf16) with((bf16_t*)nullptr);
    else with((float*)nullptr);
}
// The rows' last workgroup adds up the pairs where few are counted, one after the other: 1 600 rows 11.3 us, two launches 12.4; 800 rows
// 11.1 and 12.5; but 6 400 rows 30.9 and 12.8.  Its 16 groups of lanes have at most two sequences each then.  What is saved is the launch; where the
// rows take longer than that, the second launch is ready before they end: 1 600 rows of 30 000 logits 24.4 and 22.4.
constexpr int kLastRows = 1600, kLastPairs = 16, kLastLogits = 1 << 23;

}  // namespace

hipError_t launch_preference_forward(const PreferenceArgs& a, bool bf16, hipStream_t s) {
    const bool last = a.rows > 0 && a.rows <= kLastRows && a.pairs <= kLastPairs && (int64_t)a.rows * a.vocab <= kLastLogits;
    if (a.rows > 0) {
        by_row(a, bf16, [&](auto* t, auto strip) {
            typedef std::remove_pointer_t<decltype(t)> T;
            constexpr int S = decltype(strip)::value;
            const dim3 grid((a.rows + 3) / 4);
            if (last) preference_rows_kernel<T, S, true><<<grid, 256, 0, s>>>(a);
            else preference_rows_kernel<T, S, false><<<grid, 256, 0, s>>>(a);
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || last) return e;
    }
    preference_pairs_kernel<<<1, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_preference_backward(const PreferenceArgs& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    by_row(a, bf16, [&](auto* t, auto strip) {
        preference_gradient_kernel<std::remove_pointer_t<decltype(t)>, decltype(strip)::value><<<dim3((a.rows + 3) / 4), 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace aed
