// The divergence of rows of logits z from a teacher's largest logits, and its gradient by z.
//
//   L_r = T^2 (sum_k q_k log(q_k / p_k) + q_R log(q_R / p_R)),  p = softmax(z / T), R: all ids that are not in the row's list
//   dz_i = w_r T (p_i - q_i) in the list,  w_r T p_i (1 - q_R / p_R) outside of it
//
// Bound by memory: forward reads the logits once, backward reads them again and writes as much.  What the list needs (some 32 elements of
// thousands) is made in forward in 64 bits where it is a small difference of large numbers, its gradients too; backward writes p's multiple
// everywhere and then the list's own.  p_R is the sum over what is not in the list, found by a bit for each id in LDS, and never a difference to 1: of
// a student that is sure of the list it is 1e-10 and less.  What lies outside is taken relative to its own largest logit, so that p_i / p_R keeps its digits too.
// 8448 rows of 4096 in bfloat16, lists of 32 and others: forward 22 us (3.2 TB/s; exponentials and the list's 64 bits, between them, cost as much as the reading),
// sum of the rows 4, backward 25 (5.6 TB/s: much of the logits is still in the memory-side cache).  2048 rows of 33000 in float32: 48 us (5.6 TB/s) and 90 (6.0).
#include <algorithm>

#include "vocab_rows.h"

namespace aed {

namespace {

// Largest logit and the sum of 2^((z - top) scale)
struct Partial {
    float top;
    double sum;
};

// 2^y, minus infinity and NaN as they are
__device__ __forceinline__ double exactly(const Pow2& pow2, double y) { return y != y ? y : pow2(y); }
constexpr int kMarks = 8192;  // ids of a list that fall on the same of so many bits may be the same

}  // namespace

// W wavefronts a row, S vectors of it a thread at once, E entries of the list a lane.  OTHERS: what is not in the list is a class of its own.  LDS: a bit for
// each id, or for the last digits of each.
template <typename T, int W, int S, int E, bool OTHERS> __global__ __launch_bounds__(64 * W) void distill_rows_kernel(DistillArgs a) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::n, kThreads = 64 * W;
    extern __shared__ uint32_t listed[];
    __shared__ Partial parts[W];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.top, vocab = a.z.vocab;
    float* const stats = a.stats + (int64_t)r * (K + 2);
    // the list: entry 64 i + lane
    float value[E], at[E];
    int id[E];
    bool valid[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int k = min(64 * i + lane, K - 1);
        value[i] = a.values[(int64_t)r * K + k];
        id[i] = a.ids[(int64_t)r * K + k];
    }
    if (a.weights && a.weights[r] == 0.f) {
        if (tid == 0) a.row_loss[r] = 0.f;
        return;
    }
    const T* const z = static_cast<const T*>(a.z.data) + r * a.z.stride;
    const int vecs = (vocab + N - 1) / N, steps = (vecs + kThreads * S - 1) / (kThreads * S);
    V x[S];
    auto read = [&](int step) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int first = ((step * S + i) * kThreads + tid) * N;
            if (((step * S + i) * kThreads + kThreads) * N <= vocab) x[i] = *reinterpret_cast<const typename RowVec<T>::any*>(z + first);
            else x[i] = row_vec(z, first, vocab);
        }
    };
    read(0);
#pragma unroll
    for (int i = 0; i < E; ++i) {
        valid[i] = 64 * i + lane < K && (unsigned)id[i] < (unsigned)vocab && value[i] != -kInf;
        if (!valid[i]) id[i] = -1;
        at[i] = -kInf;
        if (valid[i] && wave == 0) at[i] = to_f32(z[id[i]]);
    }
    bool twice = false;  // an id may stand twice in the list
    {
        const int words = (min(vocab, OTHERS ? kMostVocab : kMarks) + 31) / 32;
        for (int i = tid; i < words; i += kThreads) listed[i] = 0;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int mark = OTHERS ? id[i] : id[i] & (kMarks - 1);
                if (valid[i]) twice |= atomicOr(&listed[mark >> 5], 1u << (mark & 31)) >> (mark & 31) & 1;
            }
        }
        if (OTHERS) __syncthreads();
    }

    // The row: all of it, or what is not in the list.  A divergence is a small difference of logarithms, so its sum has to be better than its terms: the
    // scale has two parts (the second above 0, so that minus infinity stays), and where lanes come together there are 64 bits.  One part alone made rows' losses
    // at T = 4 wrong by 3e-5 of themselves.
    const Pow2 pow2;
    const double c = a.scale_d;
    const float scale = a.scale, scale_low = a.scale_low;
    float lane_top = -kInf, lane_sum = 0.f;  // the sum is relative to 2^lane_base
    double lane_base = -(double)kInf;
    for (int step = 0; step < steps; ++step) {
        float y[S][N], top = lane_top;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            uint32_t bits = 0;
            if constexpr (OTHERS) {
                const int first = ((step * S + i) * kThreads + tid) * N;
                if (first < vocab) bits = listed[first >> 5] >> (first & 31) << (first - vec_begin<N>(first, vocab));
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                y[i][e] = to_f32((T)x[i][e]);
                if constexpr (OTHERS) {  // minus infinity under the bit
                    const uint32_t mask = (int)(bits << (31 - e)) >> 31;
                    y[i][e] = bits_f32((__builtin_bit_cast(uint32_t, y[i][e]) & ~mask) | (mask & 0xff800000u));
                }
                top = fmaxf(top, y[i][e]);
            }
        }
        if (step + 1 < steps) read(step + 1);
        const float to = top == -kInf ? 0.f : top, product = to * scale;
        const bool wide = __any(fabsf(product) > 0x1p24f);  // the product's own rounding may be some powers of two
        const double base = wide ? (double)to * c : (double)product;
        float sum = 0.f;
        if (!wide) {
#pragma unroll
            for (int i = 0; i < S; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) sum += __builtin_amdgcn_exp2f(fmaf(y[i][e], scale_low, fmaf(y[i][e], scale, -product)));
        } else {
#pragma unroll
            for (int i = 0; i < S; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) sum += __builtin_amdgcn_exp2f(fmaf(y[i][e] - to, scale_low, (y[i][e] - to) * scale));
        }
        lane_sum = fmaf(lane_sum, __builtin_amdgcn_exp2f((float)(lane_base - base)), sum);
        lane_top = top;
        lane_base = top == -kInf ? -(double)kInf : base;
    }
    Partial mine;
    mine.top = wave_max(lane_top);
    mine.sum = wave_sum((double)lane_sum * pow2(lane_base - (mine.top == -kInf ? 0.0 : (double)mine.top * c)));
    if constexpr (W > 1) {
        if (lane == 0) parts[wave] = mine;
        __syncthreads();
        if (wave != 0) return;
        for (int i = 1; i < W; ++i) {
            const Partial other = parts[i];
            const float top = fmaxf(mine.top, other.top);
            const double to = top == -kInf ? 0.0 : (double)top;
            mine.sum = mine.sum * pow2(((double)mine.top - to) * c) + other.sum * pow2(((double)other.top - to) * c);
            mine.top = top;
        }
    }

    // the list against the row, by one wavefront, in 64 bits; logarithms to base 2
    const double rest = OTHERS ? (double)a.rest[r] * kLog2eD : -(double)kInf;
    float value_top = -kInf, at_top = -kInf;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        value_top = fmaxf(value_top, valid[i] ? value[i] : -kInf);
        at_top = fmaxf(at_top, at[i]);
    }
    value_top = wave_max(value_top);
    at_top = wave_max(at_top);
    const double lead = fmax((double)value_top * c, rest);
    bool entry = false;
#pragma unroll
    for (int i = 0; i < E; ++i) entry = entry || valid[i];
    if (!__any(entry) && !(fabs(rest) < (double)kInf)) {  // neither an entry nor a finite rest; an entry that is NaN is one
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (64 * i + lane < K) stats[2 + 64 * i + lane] = kLeftOut;
        if (lane == 0) {
            stats[0] = stats[1] = 0.f;
            a.row_loss[r] = 0.f;
        }
        return;
    }
    // the teacher's, and the student's relative to its largest
    const bool some = mine.top > -kInf;  // of what the row gave
    const float top = OTHERS ? fmaxf(mine.top, at_top) : mine.top;
    const double to = top == -kInf ? 0.0 : (double)top, row_top = some ? ((double)mine.top - to) * c : 0.0;
    double log_q[E], q[E], same[E], p[E], n = 0, total = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        log_q[i] = (double)value[i] * c - lead;
        q[i] = valid[i] ? exactly(pow2, log_q[i]) : 0.0;
        p[i] = valid[i] ? exactly(pow2, ((double)at[i] - to) * c) : 0.0;
        n += q[i];
        total += p[i];
    }
    n = wave_sum(n);
    // lane 0: the rest's part of n, others: what the row's sum is relative to the student's largest
    const double uniform = exactly(pow2, lane == 0 ? rest - lead : row_top);
    const double q_others = OTHERS ? lane_of(uniform, 0) : 0.0, shift = lane_of(uniform, 1), others = mine.sum * shift;
    n += q_others;
    if (__any(twice)) {  // entries of one id share what they have; the first of them counts for p
        for (int i = 0; i < E; ++i) same[i] = 0;
        total = 0;
        bool again[E];
#pragma unroll
        for (int i = 0; i < E; ++i) again[i] = false;
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (k >> 6 != j) continue;
                const int other = __builtin_amdgcn_readlane(id[j], k & 63);
                const double more = lane_of(q[j], k & 63);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    same[i] += other == id[i] ? more : 0.0;
                    again[i] |= other == id[i] && k < 64 * i + lane;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) total += again[i] ? 0.0 : p[i];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) same[i] = q[i];
    }
    total = OTHERS ? wave_sum(total) + others : others;
    // lane 0: of n, 1: of the student's sum, 2: of what the row gave
    const double of = lane == 0 ? n : lane == 1 ? total : mine.sum;
    const double inverse = of > 0 ? 1 / of : of == 0 ? 0 : of, log_of = of == 0 ? 0.0 : log2_of(pow2, of);  // NaN stays; without any logit every p is 0
    const double n_inverse = lane_of(inverse, 0), total_inverse = lane_of(inverse, 1), log_n = lane_of(log_of, 0), log_total = lane_of(log_of, 1);
    double row = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        q[i] *= n_inverse;
        if (q[i] != 0) row += q[i] * (log_q[i] - log_n - (((double)at[i] - to) * c - log_total));
    }
    row = wave_sum(row);
    double outside = shift * total_inverse;  // p_i = 2^((z_i - top) scale) of this, less what p_R takes
    if constexpr (OTHERS) {
        const double q_rest = q_others * n_inverse;
        const double log_others = some ? lane_of(log_of, 2) + row_top : -(double)kInf;
        if (q_rest != 0) row += q_rest * (rest - lead - log_n - (log_others - log_total));
        outside -= q_rest * lane_of(inverse, 2);
    }
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (64 * i + lane < K) stats[2 + 64 * i + lane] = valid[i] ? (float)(p[i] * total_inverse - same[i] * n_inverse) : kLeftOut;
    if (lane == 0) {
        stats[0] = some ? mine.top : 0.f;
        stats[1] = (float)(some ? outside : mine.sum);  // 0, or NaN if the row has one
        a.row_loss[r] = (float)(a.factor * row);
    }
}

// One workgroup adds up the rows, in one order
__global__ __launch_bounds__(1024) void distill_loss_kernel(DistillArgs a) {
    const int tid = threadIdx.x;
    __shared__ double part[16];
    double v = 0;
    for (int first = tid; first < a.z.rows; first += 16384) {
        float w[16], l[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = min(first + 1024 * i, a.z.rows - 1);
            w[i] = a.weights ? a.weights[r] : 1.f;
            l[i] = a.row_loss[r];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) v += w[i] == 0.f || first + 1024 * i >= a.z.rows ? 0.0 : (double)w[i] * (double)l[i];
    }
    v = wave_sum(v);
    if ((tid & 63) == 0) part[tid >> 6] = v;
    __syncthreads();
    if (tid == 0) {
        v = 0;
        for (int i = 0; i < 16; ++i) v += part[i];
        a.loss[0] = (float)(a.weights || a.z.rows == 0 ? v : v / (double)a.z.rows);
    }
}

// W wavefronts a row, S vectors read before the first is written.  The list's elements are written when the row's have arrived: the same addresses, by other
// lanes.  Rows are taken from the last one on: those that forward has read last are still in the memory-side cache.  STREAM: gradients that it could not hold
// anyway pass it by, and leave the logits there.
template <typename T, int W, int S, bool STREAM> __global__ __launch_bounds__(64 * W) void distill_gradient_kernel(DistillArgs a) {
    typedef typename RowVec<T>::type V;
    constexpr int N = RowVec<T>::n, kThreads = 64 * W;
    const int r = gridDim.x - 1 - blockIdx.x, tid = threadIdx.x, K = a.top, vocab = a.z.vocab;
    const T* const z = static_cast<const T*>(a.z.data) + r * a.z.stride;
    T* const d = static_cast<T*>(a.d_logits) + r * a.d_stride;
    const float w = a.weights ? a.weights[r] : 1.f / (float)a.z.rows;
    const float* const stats = a.stats + (int64_t)r * (K + 2);
    const int vecs = (vocab + N - 1) / N;
    // the vector's own elements, at the row's end too
    auto put = [&](int v, const V& y) {
        const int first = v * N;
        if (first + N <= vocab) {
            if constexpr (STREAM) __builtin_nontemporal_store(y, reinterpret_cast<typename RowVec<T>::any*>(d + first));
            else *reinterpret_cast<typename RowVec<T>::any*>(d + first) = y;
            return;
        }
        const int begin = vec_begin<N>(first, vocab);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (begin + e >= first && begin + e < vocab) d[begin + e] = y[e];
    };
    // Nothing outside of the list: of a row that forward has left out, the logits may be anything, and are not looked at.
    const bool none = w == 0.f || stats[1] == 0.f;
    if (none)
        for (int v = tid; v < vecs; v += kThreads) put(v, (V)(from_f32<T>(0.f)));
    if (w == 0.f) return;
    const float scale = (float)a.scale_d, slope = w * a.temperature * (a.d_loss ? a.d_loss[0] : 1.f);
    const float s0 = stats[0], s1 = slope * stats[1];
    for (int v0 = none ? vecs : tid; v0 < vecs; v0 += kThreads * S) {
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
        const int id = a.ids[(int64_t)r * K + k];
        if (g != kLeftOut && (unsigned)id < (unsigned)vocab) d[id] = from_f32<T>(slope * g);
    }
}

namespace {

template <typename T, int W, int S, int E> hipError_t launch_rows_as(const DistillArgs& a, hipStream_t s) {
    const size_t words = (size_t)(std::min(a.z.vocab, a.rest ? kMostVocab : kMarks) + 31) / 32;
    if (a.rest) distill_rows_kernel<T, W, S, E, true><<<dim3(a.z.rows), dim3(64 * W), words * 4, s>>>(a);
    else distill_rows_kernel<T, W, S, E, false><<<dim3(a.z.rows), dim3(64 * W), words * 4, s>>>(a);
    return hipGetLastError();
}
template <typename T, int E> hipError_t launch_rows_of(const DistillArgs& a, hipStream_t s) {
    // by one wavefront, as long as it has a row of a few vectors a lane: 8448 rows of 4096 in bfloat16, both directions, 51 us, and 64 by four; 2048 of 33000 in float32
    // 184 by one, 147 by four
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    if (vecs <= 64 * 2) return launch_rows_as<T, 1, 2, E>(a, s);
    if (vecs <= 64 * 16) return launch_rows_as<T, 1, 4, E>(a, s);
    return launch_rows_as<T, 4, 4, E>(a, s);
}
// Half of the memory-side cache.  Forward and backward, 2048 rows of 33000 in float32 (270 MB) 183 -> 145 us by both the order and the stores, 28864 of 4096 in
// bfloat16 (236 MB) 155 -> 130, and 283 -> 259 with a pass that reads the gradients behind it; 8448 of 4096 (69 MB) 51 -> 49, and 93 -> 94.
constexpr int64_t kStreamBytes = 1 << 27;

template <typename T, int W> hipError_t launch_gradient_as(const DistillArgs& a, hipStream_t s) {
    if ((int64_t)a.z.rows * a.z.vocab * (int64_t)sizeof(T) > kStreamBytes) distill_gradient_kernel<T, W, 8, true><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    else distill_gradient_kernel<T, W, 8, false><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t launch_gradient_of(const DistillArgs& a, hipStream_t s) {
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    return vecs <= 64 * 16 ? launch_gradient_as<T, 1>(a, s) : launch_gradient_as<T, 4>(a, s);
}

}  // namespace

hipError_t launch_distill_forward(const DistillArgs& a, bool bf16, hipStream_t s) {
    if (a.z.rows > 0) {
        const hipError_t e = a.top <= 64 ? bf16 ? launch_rows_of<bf16_t, 1>(a, s) : launch_rows_of<float, 1>(a, s)
                                        : bf16 ? launch_rows_of<bf16_t, 2>(a, s) : launch_rows_of<float, 2>(a, s);
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
