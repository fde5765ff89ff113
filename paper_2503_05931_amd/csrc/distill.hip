// The divergence of rows of logits z from a teacher's largest logits, and its gradient by z.
//
//   L_r = T^2 (sum_k q_k log(q_k / p_k) + q_R log(q_R / p_R)),  p = softmax(z / T), R: all ids that are not in the row's list
//   dz_i = w_r T (p_i - q_i) in the list,  w_r T p_i (1 - q_R / p_R) outside of it
//
// Bound by memory: forward reads the logits once, backward reads them again and writes as much.  What the list needs (some 32 elements of
// thousands) is made in forward in 64 bits where it is a small difference of large numbers, its gradients too; backward writes p's multiple
// everywhere and then the list's own.  p_R is the sum over what is not in the list, found by a bit for each id in LDS, and never a difference to 1: of
// a student that is sure of the list it is 1e-10 and less.  What lies outside is taken relative to its own largest logit, so that p_i / p_R keeps its digits too.
#include "vocab_rows.h"

namespace aed {

namespace {

// (maximum, sum of exponentials relative to it): of two parts
struct Partial {
    float m, l;
};
__device__ __forceinline__ Partial joined(Partial a, Partial b, float scale) {
    const float m = fmaxf(a.m, b.m), base = m == -kInf ? 0.f : m;
    return Partial{m, a.l * __builtin_amdgcn_exp2f((a.m - base) * scale) + b.l * __builtin_amdgcn_exp2f((b.m - base) * scale)};
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int by = 1; by < 64; by *= 2) v += __shfl_xor(v, by);
    return v;
}

constexpr int kPer = kMostTop / 64;  // entries of a lane

}  // namespace

// W wavefronts a row, S vectors of it a thread at once.  OTHERS: what is not in the list is a class of its own.  LDS: a bit for each id, with OTHERS.
template <typename T, int W, int S, bool OTHERS> __global__ __launch_bounds__(64 * W) void distill_rows_kernel(DistillArgs a) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::n, kThreads = 64 * W;
    extern __shared__ uint32_t listed[];
    __shared__ Partial parts[W];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.top, vocab = a.z.vocab;
    float* const stats = a.stats + (int64_t)r * (K + 2);
    if (a.weights && a.weights[r] == 0.f) {
        if (tid == 0) a.row_loss[r] = 0.f;
        return;
    }
    const T* const z = static_cast<const T*>(a.z.data) + r * a.z.stride;
    const float scale = (float)(kLog2eD / (double)a.temperature);

    // the list: entry 64 i + lane
    float value[kPer], at[kPer];
    int id[kPer];
    bool valid[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int k = 64 * i + lane;
        value[i] = -kInf;
        id[i] = -1;
        at[i] = -kInf;
        if (k < K) {
            value[i] = a.values[(int64_t)r * K + k];
            id[i] = a.ids[(int64_t)r * K + k];
        }
        valid[i] = (unsigned)id[i] < (unsigned)vocab && value[i] != -kInf;
        if (!valid[i]) id[i] = -1;
        else if (wave == 0) at[i] = to_f32(z[id[i]]);
    }
    if constexpr (OTHERS) {
        for (int i = tid; i < (vocab + 31) / 32; i += kThreads) listed[i] = 0;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (valid[i]) atomicOr(&listed[id[i] >> 5], 1u << (id[i] & 31));
        }
        __syncthreads();
    }

    // the row: all of it, or what is not in the list
    Partial mine{-kInf, 0.f};
    const int vecs = (vocab + N - 1) / N;
    for (int v0 = tid; v0 < (vecs + kThreads * S - 1) / (kThreads * S) * (kThreads * S); v0 += kThreads * S) {
        V x[S];
#pragma unroll
        for (int i = 0; i < S; ++i) x[i] = row_vec(z, (v0 + kThreads * i) * N, vocab);
        float y[S][N], top = mine.m;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            uint32_t bits = 0;
            if constexpr (OTHERS) {
                const int first = (v0 + kThreads * i) * N;
                if (first < vocab) bits = listed[first >> 5] >> (first & 31) << (first - vec_begin<N>(first, vocab));
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                y[i][e] = to_f32((T)x[i][e]);
                if constexpr (OTHERS) y[i][e] = bits >> e & 1 ? -kInf : y[i][e];
                top = fmaxf(top, y[i][e]);
            }
        }
        const float base = top == -kInf ? 0.f : top;
        mine.l *= __builtin_amdgcn_exp2f((mine.m - base) * scale);
        mine.m = top;
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) mine.l += __builtin_amdgcn_exp2f((y[i][e] - base) * scale);
    }
    {
        const float top = wave_max(mine.m), base = top == -kInf ? 0.f : top;
        mine = Partial{top, wave_sum(mine.l * __builtin_amdgcn_exp2f((mine.m - base) * scale))};
    }
    if constexpr (W > 1) {
        if (lane == 0) parts[wave] = mine;
        __syncthreads();
        if (wave != 0) return;
        for (int i = 1; i < W; ++i) mine = joined(mine, parts[i], scale);
    }

    // the list against the row, by one wavefront
    const double c = 1.0 / (double)a.temperature;
    const float rest = OTHERS ? a.rest[r] : -kInf;
    float value_top = -kInf, at_top = -kInf;
    bool again[kPer];  // the id stands further in front, too
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        value_top = fmaxf(value_top, valid[i] ? value[i] : -kInf);
        at_top = fmaxf(at_top, at[i]);
        again[i] = false;
    }
    value_top = wave_max(value_top);
    at_top = wave_max(at_top);
    const double lead = fmax((double)value_top * c, (double)rest);
    if (lead == -(double)kInf) {  // neither an entry nor a rest
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (64 * i + lane < K) stats[2 + 64 * i + lane] = kLeftOut;
        if (lane == 0) {
            stats[0] = stats[1] = 0.f;
            a.row_loss[r] = 0.f;
        }
        return;
    }
    // the teacher's
    double log_q[kPer], q[kPer], n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        log_q[i] = (double)value[i] * c - lead;
        q[i] = valid[i] ? exp(log_q[i]) : 0.0;
        n += q[i];
    }
    n = wave_sum_d(n);
    if constexpr (OTHERS) n += exp((double)rest - lead);
    const double log_n = log(n);
    double same[kPer];  // q's sum over the entries of the id
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        log_q[i] -= log_n;
        q[i] = valid[i] ? q[i] / n : 0.0;
        same[i] = q[i];
    }
    bool any = false;
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (k >> 6 != j) continue;
            const int other = __builtin_amdgcn_readlane(id[j], k & 63);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                again[i] |= other == id[i] && k < 64 * i + lane;
                any |= other == id[i] && k != 64 * i + lane && valid[i];
            }
        }
    }
    if (__any(any)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) same[i] = 0;
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (k >> 6 != j) continue;
                const int other = __builtin_amdgcn_readlane(id[j], k & 63);
                const double more = __shfl(q[j], k & 63);
#pragma unroll
                for (int i = 0; i < kPer; ++i) same[i] += other == id[i] ? more : 0.0;
            }
        }
    }
    // the student's
    const float top = OTHERS ? fmaxf(mine.m, at_top) : mine.m;
    const double base = top == -kInf ? 0.0 : (double)top;
    double e[kPer], total = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        e[i] = valid[i] ? exp(((double)at[i] - base) * c) : 0.0;
        total += again[i] ? 0.0 : e[i];
    }
    const double shift = exp((mine.m == -kInf ? 0.0 : (double)mine.m - base) * c), others = (double)mine.l * shift;
    total = OTHERS ? wave_sum_d(total) + others : others;
    const double log_total = total == 0 ? 0.0 : log(total);  // no logit at all: every p is 0
    double row = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (q[i] != 0) row += q[i] * (log_q[i] - (((double)at[i] - base) * c - log_total));
    row = wave_sum_d(row);
    const double inverse = total > 0 ? 1 / total : total == 0 ? 0 : total;  // NaN stays
    const bool some = mine.m > -kInf;  // outside of the list: p_i = exp((z_i - s0) / T) s1, less what p_R takes
    double outside = shift * inverse;
    if constexpr (OTHERS) {
        const double log_rest = (double)rest - lead - log_n, q_rest = exp(log_rest);
        const double log_others = some ? log((double)mine.l) + ((double)mine.m - base) * c : -(double)kInf;
        if (q_rest != 0) row += q_rest * (log_rest - (log_others - log_total));
        outside -= q_rest / (double)mine.l;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (64 * i + lane < K) stats[2 + 64 * i + lane] = valid[i] ? (float)(e[i] * inverse - same[i]) : kLeftOut;
    if (lane == 0) {
        stats[0] = some ? mine.m : 0.f;
        stats[1] = some ? (float)outside : 0.f;
        a.row_loss[r] = (float)((double)a.temperature * (double)a.temperature * row);
    }
}

// One workgroup adds up the rows, in one order
__global__ __launch_bounds__(1024) void distill_loss_kernel(DistillArgs a) {
    const int tid = threadIdx.x;
    __shared__ double part[16];
    double v = 0;
    for (int r = tid; r < a.z.rows; r += 1024) {
        const float w = a.weights ? a.weights[r] : 1.f;
        v += w == 0.f ? 0.0 : (double)w * (double)a.row_loss[r];
    }
    v = wave_sum_d(v);
    if ((tid & 63) == 0) part[tid >> 6] = v;
    __syncthreads();
    if (tid == 0) {
        v = 0;
        for (int i = 0; i < 16; ++i) v += part[i];
        a.loss[0] = (float)(a.weights || a.z.rows == 0 ? v : v / (double)a.z.rows);
    }
}

// W wavefronts a row, S vectors read before the first is written.  The list's elements are written when the row's have arrived: the same addresses, by other
// lanes.
template <typename T, int W, int S> __global__ __launch_bounds__(64 * W) void distill_gradient_kernel(DistillArgs a) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::n, kThreads = 64 * W;
    const int r = blockIdx.x, tid = threadIdx.x, K = a.top, vocab = a.z.vocab;
    const T* const z = static_cast<const T*>(a.z.data) + r * a.z.stride;
    T* const d = static_cast<T*>(a.d_logits) + r * a.d_stride;
    const float w = a.weights ? a.weights[r] : 1.f / (float)a.z.rows;
    const float* const stats = a.stats + (int64_t)r * (K + 2);
    const int vecs = (vocab + N - 1) / N;
    // the vector's own elements, at the row's end too
    auto put = [&](int v, const V& y) {
        const int first = v * N;
        if (first + N <= vocab) {
            *reinterpret_cast<typename RowVec<T>::any*>(d + first) = y;
            return;
        }
        const int begin = vec_begin<N>(first, vocab);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (begin + e >= first && begin + e < vocab) d[begin + e] = y[e];
    };
    if (w == 0.f) {
        for (int v = tid; v < vecs; v += kThreads) put(v, (V)(from_f32<T>(0.f)));
        return;
    }
    const float scale = (float)(kLog2eD / (double)a.temperature), slope = w * a.temperature * (a.d_loss ? a.d_loss[0] : 1.f);
    const float s0 = stats[0], s1 = slope * stats[1];
    for (int v0 = tid; v0 < vecs; v0 += kThreads * S) {
        V x[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int first = (v0 + kThreads * i) * N;
            if (first < vocab) x[i] = row_vec(z, first, vocab);
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            V y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = from_f32<T>(s1 * __builtin_amdgcn_exp2f((to_f32((T)x[i][e]) - s0) * scale));
            if (v0 + kThreads * i < vecs) put(v0 + kThreads * i, y);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (W > 1) __syncthreads();
    for (int k = tid; k < K; k += kThreads) {
        const float g = stats[2 + k];
        if (g != kLeftOut) d[a.ids[(int64_t)r * K + k]] = from_f32<T>(slope * g);
    }
}

namespace {

template <typename T, int W, int S> hipError_t launch_rows_as(const DistillArgs& a, hipStream_t s) {
    if (a.rest) distill_rows_kernel<T, W, S, true><<<dim3(a.z.rows), dim3(64 * W), (size_t)(a.z.vocab + 31) / 32 * 4, s>>>(a);
    else distill_rows_kernel<T, W, S, false><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t launch_rows_of(const DistillArgs& a, hipStream_t s) {
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    if (vecs <= 64 * 2) return launch_rows_as<T, 1, 2>(a, s);
    if (vecs <= 64 * 16) return launch_rows_as<T, 1, 8>(a, s);
    return launch_rows_as<T, 4, 8>(a, s);
}
template <typename T> hipError_t launch_gradient_of(const DistillArgs& a, hipStream_t s) {
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    if (vecs <= 64 * 16) distill_gradient_kernel<T, 1, 8><<<dim3(a.z.rows), dim3(64), 0, s>>>(a);
    else distill_gradient_kernel<T, 4, 8><<<dim3(a.z.rows), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill_forward(const DistillArgs& a, bool bf16, hipStream_t s) {
    if (a.z.rows > 0) {
        const hipError_t e = bf16 ? launch_rows_of<bf16_t>(a, s) : launch_rows_of<float>(a, s);
        if (e != hipSuccess) return e;
    }
    distill_loss_kernel<<<1, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_distill_backward(const DistillArgs& a, bool bf16, hipStream_t s) {
    if (a.z.rows == 0) return hipSuccess;
    return bf16 ? launch_gradient_of<bf16_t>(a, s) : launch_gradient_of<float>(a, s);
}

}  // namespace aed
