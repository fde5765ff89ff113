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

namespace aed {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kStrip = 8;  // vectors of a row that a lane holds at once

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

// One wavefront a row, eight vectors of it at once: 5.1 TB/s.
template <typename T> __global__ __launch_bounds__(256) void preference_rows_kernel(PreferenceArgs a) {
    typedef typename Vec<T>::type V;
    constexpr int N = Vec<T>::n;
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.rows) return;
    const int label = a.labels[row];
    if (!scored(label, a.vocab)) {
        if (lane == 0) {
            a.gain[row] = 0.f;
            a.lse[row] = float2{0.f, 0.f};
        }
        return;
    }
    const T* const z = static_cast<const T*>(a.logits) + row * a.row_stride;
    const RowParts<T> part(z, a.vocab);
    const V* const zv = reinterpret_cast<const V*>(z + part.head);
    float m = -__builtin_inff(), l = 0.f;
    const int at = part.loose(lane, a.vocab);
    if (at >= 0) {
        m = to_f32(z[at]);
        l = m == -__builtin_inff() ? 0.f : 1.f;
    }
    for (int v0 = lane; v0 < part.vecs; v0 += 64 * kStrip) {
        V x[kStrip];
#pragma unroll
        for (int i = 0; i < kStrip; ++i) x[i] = zv[min(v0 + 64 * i, part.vecs - 1)];
        float y[kStrip][N], top = m;
#pragma unroll
        for (int i = 0; i < kStrip; ++i) {
            const bool there = v0 + 64 * i < part.vecs;
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
        for (int i = 0; i < kStrip; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) l += __builtin_amdgcn_exp2f((y[i][e] - base) * kLog2e);
    }
    const float top = wave_max(m), base = top == -__builtin_inff() ? 0.f : top;
    l = wave_sum(l * __builtin_amdgcn_exp2f((m - base) * kLog2e));
    if (lane == 0) {
        const float log_l = kLn2 * __builtin_amdgcn_logf(l);
        a.lse[row] = float2{top, log_l};
        a.gain[row] = (to_f32(z[label]) - top) - log_l - a.ref[row];
    }
}

// -log sigmoid(x)
__device__ __forceinline__ float loss_of(float x) { return fmaxf(-x, 0.f) + log1pf(expf(-fabsf(x))); }

// One workgroup: sixteen lanes add up a sequence, 64 sequences at once, then the pairs' losses are added.
__global__ __launch_bounds__(1024) void preference_pairs_kernel(PreferenceArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = threadIdx.x & 15;
    __shared__ float part[16];
    float mine = 0.f;
    for (int s = threadIdx.x >> 4; s < 2 * a.pairs; s += 64) {  // both sequences of a pair are a wavefront's
        const int first = a.seq_start[s], end = a.seq_start[s + 1];
        float v = 0.f;
#pragma unroll 8
        for (int i = first + sub; i < end; i += 16) v += a.gain[i];
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
        for (int i = 0; i < 16; ++i) v += part[i];
        a.loss[0] = v / (float)a.pairs;
    }
}

// One wavefront a row; row t's gradient is slope (onehot - softmax).  Eight vectors are read before the first is written: 21.8 us, 22.6
// one by one.
template <typename T> __global__ __launch_bounds__(256) void preference_gradient_kernel(PreferenceArgs a) {
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
    for (int v0 = lane; v0 < part.vecs; v0 += 64 * kStrip) {
        V x[kStrip];
#pragma unroll
        for (int i = 0; i < kStrip; ++i) {
            const T* const from = z + part.head + min(v0 + 64 * i, part.vecs - 1) * N;
            if (same) x[i] = *reinterpret_cast<const V*>(from);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] = from[e];
            }
        }
#pragma unroll
        for (int i = 0; i < kStrip; ++i) {
            const int v = v0 + 64 * i;
            V y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = gradient(to_f32((T)x[i][e]), part.head + v * N + e);
            if (v < part.vecs) dv[v] = y;
        }
    }
}

hipError_t launch_preference_forward(const PreferenceArgs& a, bool bf16, hipStream_t s) {
    if (a.rows > 0) {
        const dim3 grid((a.rows + 3) / 4);
        if (bf16) preference_rows_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
        else preference_rows_kernel<float><<<grid, 256, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    preference_pairs_kernel<<<1, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_preference_backward(const PreferenceArgs& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const dim3 grid((a.rows + 3) / 4);
    if (bf16) preference_gradient_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
    else preference_gradient_kernel<float><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace aed
