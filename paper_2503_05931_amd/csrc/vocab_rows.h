// Device side of a row of logits: reading it at any alignment, its order (larger first, equal ones by id), and the
// search for a place in that order.
#pragma once

#include <limits.h>

#include "common.h"
#include "vocab.h"

namespace aed {

constexpr float kInf = __builtin_inff();
constexpr double kLog2eD = 1.4426950408889634074;

// vectors of 16 bytes at any address that is a multiple of an element: gfx950 loads and stores those as they are
template <typename T> struct RowVec;
template <> struct RowVec<bf16_t> {
    typedef bf16x8 type;
    typedef __bf16 any __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr int n = 8;
};
template <> struct RowVec<float> {
    typedef f32x4 type;
    typedef float any __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr int n = 4;
};
// Vector v of a row of n elements begins at v N; the last one, if it is not whole, at n - N, and its elements before v N, which are the
// vector's in front of it, are left out.  So no lane branches off at a row's end, and ids rise with lanes.
template <int N> __device__ __forceinline__ int vec_begin(int id, int n) { return n >= N ? min(id, n - N) : id; }
// minus infinity in the place of what is left out
template <typename T> __device__ __forceinline__ typename RowVec<T>::type row_vec(const T* p, int id, int n) {
    constexpr int N = RowVec<T>::n;
    typename RowVec<T>::type v;
    if (n >= N) {
        const int at = min(id, n - N);
        v = *reinterpret_cast<const typename RowVec<T>::any*>(p + at);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = at + e >= id ? v[e] : from_f32<T>(-kInf);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = id + e < n ? p[id + e] : from_f32<T>(-kInf);
    }
    return v;
}

// A row that W wavefronts hold in registers, S vectors a thread; S = 0: read anew each time.  Vector v of the row is thread v % (64 W)'s.
template <typename T, int W, int S> struct Row {
    typedef typename RowVec<T>::type V;
    static constexpr int N = RowVec<T>::n, kThreads = 64 * W, kStep = kThreads * N;
    const T* p;
    int n;
    V x[S > 0 ? S : 1];
    __device__ __forceinline__ V read(int s) const {
        const int id = s * kStep + (int)threadIdx.x * N;
        if (s * kStep >= n) return (V)(from_f32<T>(-kInf));
        if ((s + 1) * kStep <= n) return *reinterpret_cast<const typename RowVec<T>::any*>(p + id);
        return row_vec(p, id, n);
    }
    __device__ __forceinline__ Row(const T* p, int n) : p(p), n(n) {}
    // the same row from memory: for what is seldom done, and would keep the registers
    __device__ __forceinline__ Row<T, W, 0> again() const { return Row<T, W, 0>(p, n); }
    __device__ __forceinline__ Row(const LogitRows& z, int row) : p(static_cast<const T*>(z.data) + row * z.stride), n(z.vocab) {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) x[s] = read(s);
        }
    }
    // f(s, first id, vector); every thread of a wavefront comes along to the last step
    template <typename F> __device__ __forceinline__ void each_vec(F f) const {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) f(s, vec_begin<N>(s * kStep + (int)threadIdx.x * N, n), x[s]);
        } else {
            for (int s = 0; s * kStep < n; ++s) f(s, vec_begin<N>(s * kStep + (int)threadIdx.x * N, n), read(s));
        }
    }
    // f(logit, id); an id may come again, or one behind the row's end, with minus infinity
    template <typename F> __device__ __forceinline__ void each(F f) const {
        each_vec([&](int, int id, const V& v) {
#pragma unroll
            for (int e = 0; e < N; ++e) f(to_f32((T)v[e]), id + e);
        });
    }
};

__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_mov<0xB1>(v));
    v = fmaxf(v, dpp_mov<0x4E>(v));
    v = fmaxf(v, dpp_mov<0x141>(v));
    v = fmaxf(v, dpp_mov<0x140>(v));
    return rows4_max(v);
}
__device__ __forceinline__ float wave_min(float v) { return -wave_max(-v); }

// 64-bit sums over a wavefront, whole numbers: in any order the same
template <int CTRL> __device__ __forceinline__ uint64_t dpp_mov64(uint64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, true);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
    v += dpp_mov64<0xB1>(v);
    v += dpp_mov64<0x4E>(v);
    v += dpp_mov64<0x141>(v);
    v += dpp_mov64<0x140>(v);
    auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    v = ((uint64_t)hi[0] << 32 | lo[0]) + ((uint64_t)hi[1] << 32 | lo[1]);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    hi = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    return ((uint64_t)hi[0] << 32 | lo[0]) + ((uint64_t)hi[1] << 32 | lo[1]);
}
// of the lanes up to this one
__device__ __forceinline__ uint64_t wave_prefix64(uint64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const uint64_t o = __shfl_up(v, by);
        if (lane >= by) v += o;
    }
    return v;
}

// The j-th largest of the lanes' values (1 <= j <= 64)
__device__ __forceinline__ float lanes_jth(float v, int j) {
    int above = 0;
#pragma unroll
    for (int l = 0; l < 64; ++l) above += bits_f32(__builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)) > v;
    return wave_min(above < j ? v : kInf);
}

// An element's place in the order
struct Place {
    float z;
    int id;
};
__device__ __forceinline__ bool before(float z, int id, float z2, int id2) { return z > z2 || (z == z2 && id < id2); }
// in the order up to `last`
__device__ __forceinline__ bool up_to(float z, int id, const Place& last) { return z > last.z || (z == last.z && id <= last.id); }

// ---- the part of a row that can hold its first elements, gathered in LDS ----
// At least `want` elements are at or above the bound: each of the wavefronts that the row fills takes the (want / wavefronts)-th largest of its lanes'
// maxima, and the least of these is the bound (no lane's maximum is counted twice).
constexpr int kList = 256;
struct List {
    int count;  // may be more than kList: then the list is cut off and of no use
    float z[kList];
    int id[kList];
};
template <int W> struct RowBounds {
    float top[W], jth[W];
};

// Every thread has the row's largest logit and the bound.
template <int W, typename R> __device__ __forceinline__ void bound_row(const R& row, int want, RowBounds<W>& lds, List& list, float& top, float& bound) {
    float m = -kInf;
    row.each([&](float z, int) { m = fmaxf(m, z); });  // NaN is passed over
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int full = max(1, min(W, row.n / (64 * R::N))), j = (want + full - 1) / full;
    const float wave_top = wave_max(m), jth = want <= 1 ? wave_top : j > 64 ? -kInf : lanes_jth(m, j);
    if constexpr (W == 1) {
        top = wave_top;
        bound = jth;
        if (lane == 0) list.count = 0;
        __syncthreads();
    } else {
        if (lane == 0) {
            lds.top[wave] = wave_top;
            lds.jth[wave] = jth;
        }
        if (threadIdx.x == 0) list.count = 0;
        __syncthreads();
        top = lds.top[0];
        bound = lds.jth[0];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            top = fmaxf(top, lds.top[i]);
            bound = i < full ? fminf(bound, lds.jth[i]) : bound;
        }
    }
    if (want <= 1) bound = top;
}
__device__ __forceinline__ void put_in(List& list, float z, int id) {
    const int at = atomicAdd(&list.count, 1);
    if (at < kList) {
        list.z[at] = z;
        list.id[at] = id;
    }
}

// ---- exact search for the last of the first elements of the order, whatever the row holds ----
// Digit by digit over histograms of 256 bins: first of the distance to the largest logit (its floating point bits: 16 bins for each power of two
// from 2^-10 to 2^6), then of the logit's own bits, then of the id's, until the bin that the border falls into has at most kList elements; those are gathered and
// compared one by one.  Elements are counted, or (WEIGHTS) their weights are added up: whole numbers, so the order of the atomic additions
// does not matter.
struct Histogram {
    uint64_t sum[256];
    uint32_t count[256];
    uint64_t before, target;
    uint32_t members;
    int bin;
    Place last;
};
__device__ __forceinline__ uint32_t falling_bits(float z) {  // larger logits, smaller bits; -0 is 0
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.f);
    return (u & 0x80000000u) ? u : ~(u | 0x80000000u);
}
__device__ __forceinline__ int distance_bin(float z, float top) {
    const uint32_t u = __builtin_bit_cast(uint32_t, z == top ? 0.f : top - z) >> 19;
    constexpr int first = (127 - 10) << 4;
    return min(max((int)u - first, 0), 255);
}

// target: for counts, how many elements the first part has; for weights, the least sum that the part up to its last element reaches; 1 or more, and
// what is more than there is counts as all.  in(z, id): elements that take part, one at least (with a weight above 0); weight(z): theirs.
template <bool WEIGHTS, typename T, int W, typename In, typename Weight>
__device__ __noinline__ Place find_last(Row<T, W, 0> row, float top, uint64_t target, Histogram& h, List& list, In in, Weight weight) {
    constexpr int kThreads = 64 * W;
    const int tid = threadIdx.x, lane = tid & 63;
    int level = 0, bin0 = 0;
    uint32_t bits = 0, id_bits = 0;  // digits found so far
    uint64_t passed = 0;             // in front of the bin
    auto member = [&](float z, int id) {
        if (!(z > -kInf) || !in(z, id)) return false;
        if (level > 0 && distance_bin(z, top) != bin0) return false;
        if (level > 1 && (falling_bits(z) ^ bits) >> (32 - 8 * min(level - 1, 4)) != 0) return false;
        return level <= 5 || ((uint32_t)id ^ id_bits) >> (24 - 8 * (level - 5)) == 0;
    };
    while (true) {
        for (int i = tid; i < 256; i += kThreads) {
            h.sum[i] = 0;
            h.count[i] = 0;
        }
        __syncthreads();
        row.each([&](float z, int id) {
            if (!member(z, id)) return;
            const int digit = level == 0   ? distance_bin(z, top)
                              : level <= 4 ? falling_bits(z) >> (32 - 8 * level) & 255
                                           : (uint32_t)id >> (24 - 8 * (level - 4)) & 255;
            atomicAdd(&h.count[digit], 1u);
            if constexpr (WEIGHTS) atomicAdd((unsigned long long*)&h.sum[digit], (unsigned long long)weight(z));
        });
        __syncthreads();
        if (tid < 64) {  // four bins a lane
            uint64_t v[4], mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) mine += v[i] = WEIGHTS ? h.sum[4 * lane + i] : h.count[4 * lane + i];
            const uint64_t through = passed + wave_prefix64(mine);
            if (level == 0) {  // there may be fewer
                target = min(target, (uint64_t)__shfl(through, 63));
                if (lane == 0) h.target = target;
            }
            uint64_t at = through - mine;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (at < target && target <= at + v[i]) {  // one bin of one lane
                    h.bin = 4 * lane + i;
                    h.before = at;
                    h.members = h.count[4 * lane + i];
                }
                at += v[i];
            }
        }
        if (tid == 0) list.count = 0;
        __syncthreads();
        const int bin = h.bin;
        passed = h.before;
        target = h.target;
        if (level == 0) bin0 = bin;
        else if (level <= 4) bits |= (uint32_t)bin << (32 - 8 * level);
        else id_bits |= (uint32_t)bin << (24 - 8 * (level - 4));
        ++level;
        if (h.members <= kList || level > 7) break;
        __syncthreads();  // all have read
    }
    row.each([&](float z, int id) {
        if (member(z, id)) put_in(list, z, id);
    });
    __syncthreads();
    const int n = min(list.count, kList);
    for (int i = tid; i < n; i += kThreads) {
        const float z = list.z[i];
        const int id = list.id[i];
        uint64_t at = passed;
        for (int j = 0; j < n; ++j)
            if (before(list.z[j], list.id[j], z, id)) at += WEIGHTS ? weight(list.z[j]) : 1;
        if (at < target && target <= at + (WEIGHTS ? weight(z) : 1)) h.last = Place{z, id};
    }
    __syncthreads();
    const Place last = h.last;
    __syncthreads();  // list and histogram may be used again
    return last;
}

}  // namespace aed
