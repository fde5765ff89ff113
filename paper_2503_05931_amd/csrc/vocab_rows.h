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
    __device__ __forceinline__ Row(const LogitRows& z, int row) : p(static_cast<const T*>(z.data) + row * z.stride), n(z.vocab) {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) x[s] = read(s);
        }
    }
    // What has been read counts as new: left to itself the compiler keeps, from one pass to the next, what it has made of each element.
    __device__ __forceinline__ void forget() {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                u32x4 u = __builtin_bit_cast(u32x4, x[s]);
                asm volatile("" : "+v"(u));
                x[s] = __builtin_bit_cast(V, u);
            }
        }
    }
    // f(s, first id, vector); every thread of a wavefront comes along to the last step
    template <typename F> __device__ __forceinline__ void each_vec(F f) const {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) f(s, vec_begin<N>(s * kStep + (int)threadIdx.x * N, n), x[s]);
        } else {
            V next = read(0);
#pragma unroll 1
            for (int s = 0; s * kStep < n; ++s) {
                const V v = next;
                if ((s + 1) * kStep < n) next = read(s + 1);
                f(s, vec_begin<N>(s * kStep + (int)threadIdx.x * N, n), v);
            }
        }
    }
    // f(s, first id, logits)
    template <typename F> __device__ __forceinline__ void each_floats(F f) const {
        each_vec([&](int s, int id, const V& v) {
            float z[N];
#pragma unroll
            for (int e = 0; e < N; ++e) z[e] = to_f32((T)v[e]);
            f(s, id, z);
        });
    }
    // f(logit, id); an id may come again, or one behind the row's end, with minus infinity
    template <typename F> __device__ __forceinline__ void each(F f) const {
        each_vec([&](int, int id, const V& v) {
#pragma unroll
            for (int e = 0; e < N; ++e) f(to_f32((T)v[e]), id + e);
        });
    }
};

// A row that is read from memory anew for each pass, in a loop of short code, the next vector asked for ahead.
template <typename T, int W> struct RowLoop {
    static constexpr int N = RowVec<T>::n, kThreads = 64 * W;
    const T* p;
    int n;
    // f(s, first id, logits)
    template <typename F> __device__ __forceinline__ void each_floats(F f) const { Row<T, W, 0>(p, n).each_floats(f); }
    // f(logit, id)
    template <typename F> __device__ __forceinline__ void each(F f) const { Row<T, W, 0>(p, n).each(f); }
};

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
// sum of doubles over a wavefront, in one order
__device__ __forceinline__ double wave_sum(double v) {
    auto as_u = [](double d) { return __builtin_bit_cast(uint64_t, d); };
    auto as_d = [](uint64_t u) { return __builtin_bit_cast(double, u); };
    v += as_d(dpp_mov64<0xB1>(as_u(v)));
    v += as_d(dpp_mov64<0x4E>(as_u(v)));
    v += as_d(dpp_mov64<0x141>(as_u(v)));
    v += as_d(dpp_mov64<0x140>(as_u(v)));
    uint64_t u = as_u(v);
    auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
    auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = as_d((uint64_t)hi[0] << 32 | lo[0]) + as_d((uint64_t)hi[1] << 32 | lo[1]);
    u = as_u(v);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
    hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    return as_d((uint64_t)hi[0] << 32 | lo[0]) + as_d((uint64_t)hi[1] << 32 | lo[1]);
}
// a shift within rows of 16 lanes (zeros come in), or a row's last lane to the rows of ROWS
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ uint32_t dpp_or0(uint32_t v) {
    return __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true);
}
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ uint64_t dpp_or0(uint64_t v) {
    return (uint64_t)dpp_or0<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | dpp_or0<CTRL, ROWS>((uint32_t)v);
}
// sum of the lanes up to this one
template <typename U> __device__ __forceinline__ U wave_prefix(U v) {
    v += dpp_or0<0x111>(v);
    v += dpp_or0<0x112>(v);
    v += dpp_or0<0x114>(v);
    v += dpp_or0<0x118>(v);
    v += dpp_or0<0x142, 0xA>(v);  // lane 15 to row 1, lane 47 to row 3
    v += dpp_or0<0x143, 0xC>(v);  // lane 31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int l) { return __builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int l) { return (uint64_t)lane_of((uint32_t)(v >> 32), l) << 32 | lane_of((uint32_t)v, l); }

// larger floats, larger bits; -0 is 0
__device__ __forceinline__ uint32_t rising_bits(float z) {
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// A bound that j of the lanes' values (VALUES each, j at most 64 VALUES) at least are not below: the j-th largest with the last 16 bits of its float cleared away,
// by halving over ballots, whose counts are the scalar unit's work.  (Sixty-four lanes read one by one: 192 vector instructions for 16.)
template <int VALUES> __device__ __forceinline__ float lanes_bound(const float (&v)[VALUES], int j) {
    uint32_t high[VALUES], t = 0;
#pragma unroll
    for (int i = 0; i < VALUES; ++i) high[i] = rising_bits(v[i]) >> 16;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < VALUES; ++i) n += __builtin_popcountll(__ballot(high[i] >= (t | 1u << bit)));
        if (n >= j) t |= 1u << bit;
    }
    const uint32_t u = t << 16;
    return t <= 0x7f ? -kInf : __builtin_bit_cast(float, (u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ double lane_of(double v, int l) { return __builtin_bit_cast(double, lane_of(__builtin_bit_cast(uint64_t, v), l)); }

// 2^y: y's nearest whole number n, and 1 + f q(f) for what is left, q of degree 8 fitted to (2^f - 1) / f on [-1/2, 1/2] for the least largest error, 1.6e-14 of
// the result.  The coefficients are kept in scalar registers, where a product can take them from.  NaN counts as minus infinity.
struct Pow2 {
    double q[9];
    __device__ __forceinline__ Pow2()
        : q{0.6931471805598853, 0.24022650695722841, 0.05550410866841879, 0.009618129181143242, 0.0013333557624782767, 0.0001540344090220312, 1.525299054241159e-05,
            1.3258330955496492e-06, 1.0148218085577417e-07} {
#pragma unroll
        for (int i = 0; i < 9; ++i) asm volatile("" : "+s"(q[i]));
    }
    __device__ __forceinline__ double operator()(double y) const {
#pragma clang fp contract(off)  // the same result wherever it is made
        y = fmax(y, -1100.0);
        const double n = rint(y), f = y - n;
        double p = q[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = fma(f, p, q[i]);
        return ldexp(fma(f, p, 1.0), (int)n);
    }
    // of several at once, step by step: an exponential is a chain of operations that each wait for the one before.  They are all made here, and not one by
    // one where they are used.
    template <int N> __device__ __forceinline__ void operator()(double (&y)[N]) const {
#pragma clang fp contract(off)
        double n[N], p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            y[e] = fmax(y[e], -1100.0);
            n[e] = rint(y[e]);
            y[e] -= n[e];
            p[e] = q[8];
        }
#pragma unroll
        for (int i = 7; i >= 0; --i)
#pragma unroll
            for (int e = 0; e < N; ++e) p[e] = fma(y[e], p[e], q[i]);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = ldexp(fma(y[e], p[e], 1.0), (int)n[e]);
#pragma unroll
        for (int e = 0; e < N; ++e) asm volatile("" : "+v"(y[e]));
    }
};

// log2 x of x > 0 that is near to what a float can be: that of the float nearest, and of what 2 to its power lacks
__device__ __forceinline__ double log2_of(const Pow2& pow2, double x) {
    const double near = __builtin_amdgcn_logf((float)x), left = x * pow2(-near) - 1;  // some 1e-7
    return near + left * (1 - 0.5 * left) * kLog2eD;
}

// An element's place in the order: of two, the one in front has the larger key
__device__ __forceinline__ uint64_t order_key(float z, int id) { return (uint64_t)rising_bits(z) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t u = key >> 32;
    return __builtin_bit_cast(float, (u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_id(uint64_t key) { return ~(uint32_t)key; }
struct Place {
    float z;
    int id;
};
// in the order up to `last`
__device__ __forceinline__ bool up_to(float z, int id, const Place& last) { return z > last.z || (z == last.z && id <= last.id); }
// minus infinity in the place of NaN: neither is in the order
__device__ __forceinline__ float in_order(float z) { return fmaxf(z, -kInf); }

// ---- the part of a row that can hold its first elements, gathered in LDS ----
// At least `want` elements are at or above the bound: each of the wavefronts that the row fills takes one that (want / wavefronts) of its lanes'
// maxima are not below, and the least of these is the bound (no lane's maximum is counted twice).  Where it is one of many lanes,
// each lane's halves or quarters have a maximum each: above all lanes' maxima are some 300 of a wavefront's elements, above half of the halves' 89.  Of several
// wavefronts the least bound lets in more than that: 128 of 32768, 2048 rows: 39 us, and 52 with one of 32 lanes.
constexpr int kList = 256;
constexpr float kMostFloat = 0x1.fffffep127f;
struct List {
    uint32_t count;  // may be more than kList: then it is cut off
    float bound;
    int id[kList];
    uint64_t key[kList];
};
template <int W> struct RowBounds {
    float top[W], bound[W];
};

// Every thread has the row's largest logit and the bound; want 0: minus infinity.
template <int W, typename R> __device__ __forceinline__ void bound_row(const R& row, int want, RowBounds<W>& lds, List& list, float& top, float& bound) {
    float m[4] = {-kInf, -kInf, -kInf, -kInf};  // of every fourth element
    row.each_floats([&](int, int, float (&z)[R::N]) {  // NaN is passed over
#pragma unroll
        for (int e = 0; e < R::N; ++e) m[e & 3] = fmaxf(m[e & 3], z[e]);
    });
    const float halves[2] = {fmaxf(m[0], m[1]), fmaxf(m[2], m[3])}, whole[1] = {fmaxf(halves[0], halves[1])};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int full = max(1, min(W, row.n / (64 * R::N))), j = (want + full - 1) / full;
    top = wave_max(whole[0]);
    bound = want == 1 ? top : want == 0 || j > 256 ? -kInf : j <= (W == 1 ? 32 : 24) ? lanes_bound(whole, j) : j <= 64 ? lanes_bound(halves, j) : lanes_bound(m, j);
    if constexpr (W > 1) {
        if (lane == 0) {
            lds.top[wave] = top;
            lds.bound[wave] = bound;
        }
        if (threadIdx.x == 0) list.count = 0;
        __syncthreads();
        top = lds.top[0];
        bound = lds.bound[0];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            top = fmaxf(top, lds.top[i]);
            bound = i < full ? fminf(bound, lds.bound[i]) : bound;
        }
        if (want == 1) bound = top;
    }
}
// a bound as gather's differences need it: finite, and -0 for 0, so that -0 less the bound is 0, whose sign says that it is not below
__device__ __forceinline__ float gather_bound(float bound) {
    bound = fminf(fmaxf(bound, -kMostFloat), kMostFloat);
    return bound == 0.f ? -0.f : bound;
}
// puts in those of each lane's vector whose sign is not set; all lanes come along
template <int N> __device__ __forceinline__ void put_in(List& list, int id, const float (&over)[N]) {
    uint32_t marks = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) marks = __builtin_amdgcn_alignbit(marks, __builtin_bit_cast(uint32_t, over[e]), 31);
    marks = ~marks << (32 - N);
    if (!__any(marks != 0)) return;
    const uint32_t mine = __builtin_popcount(marks), through = wave_prefix(mine);
    uint32_t base = 0;
    if ((threadIdx.x & 63) == 63) base = atomicAdd(&list.count, through);
    uint32_t at = lane_of(base, 63) + through - mine;
    while (marks) {
        const int e = __builtin_clz(marks);
        marks &= ~(0x80000000u >> e);
        if (at < kList) list.id[at] = id + e;
        ++at;
    }
}
// makes the first n listed elements' keys; a barrier has to follow
template <int W, typename T> __device__ __forceinline__ void read_keys(const T* p, List& list, int n) {
    for (int i = threadIdx.x; i < n; i += 64 * W) list.key[i] = order_key(in_order(to_f32(p[list.id[i]])), list.id[i]);
}
// how many of the n keys are larger
__device__ __forceinline__ int place_of(const List& list, uint64_t key, int n) {
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) place += list.key[j] > key;
    return place;
}

// Ids of the elements of which over is not negative, in no order, perhaps of some that are NaN.  over(a vector's logits) puts in the place of each a number that grows with
// it and is minus infinity for minus infinity.  Logits are read by these ids later.  A lane's elements are marked by over's signs, an instruction each (a comparison's result cannot be
// used at once), so places are handed out once a wavefront, and what is listed costs a few steps.
template <typename T, int W, int S, typename F> __device__ __forceinline__ void gather(const Row<T, W, S>& row, List& list, F over) {
    constexpr int N = RowVec<T>::n;
    if constexpr (S > 0) {
        constexpr int kMarks = (S * N + 31) / 32;
        uint32_t marks[kMarks] = {};
        row.each_floats([&](int s, int, float (&z)[N]) {
            over(z);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                uint32_t& m = marks[(s * N + e) / 32];
                m = __builtin_amdgcn_alignbit(m, __builtin_bit_cast(uint32_t, z[e]), 31);  // the sign from the right
            }
            __builtin_amdgcn_sched_barrier(0);  // one vector after the other, or all have their registers at once
        });
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < kMarks; ++i) {
            marks[i] = ~marks[i] << (S * N < 32 ? 32 - S * N : 0);
            mine += __builtin_popcount(marks[i]);
        }
        const uint32_t through = wave_prefix(mine), all = lane_of(through, 63);
        uint32_t at = through - mine;
        if constexpr (W == 1) {
            list.count = all;
        } else {
            uint32_t base = 0;
            if ((threadIdx.x & 63) == 0) base = atomicAdd(&list.count, all);
            at += lane_of(base, 0);
        }
#pragma unroll
        for (int i = 0; i < kMarks; ++i)
            while (marks[i]) {
                const int first = __builtin_clz(marks[i]), k = 32 * i + first;
                marks[i] &= ~(0x80000000u >> first);
                if (at < kList) list.id[at] = vec_begin<N>(((k / N) * 64 * W + (int)threadIdx.x) * N, row.n) + k % N;
                ++at;
            }
    } else {
        row.each_floats([&](int, int id, float (&z)[N]) {
            over(z);
            put_in(list, id, z);
        });
    }
    __syncthreads();
}

// Of a list that is cut off: the logit of its k-th element (k <= kList), a bound that k of the row are not below as well, and k / kList of those that the last one
// let in.  The list is empty then.  One row of 200 of 30000 whose lanes' maxima gave no good bound had made top-k 50 of them last 29 us, not 14.
template <int W, typename T> __device__ __forceinline__ float listed_bound(const T* p, List& list, int k) {
    read_keys<W>(p, list, kList);
    __syncthreads();
    for (int i = threadIdx.x; i < kList; i += 64 * W) {
        const uint64_t key = list.key[i];
        if (place_of(list, key, kList) == k - 1) list.bound = key_logit(key);
    }
    if (threadIdx.x == 0) list.count = 0;
    __syncthreads();
    return list.bound;
}

// ---- exact search for the last of the first elements of the order, whatever the row holds ----
// Digit by digit over histograms of 2^BITS bins: first of the distance to the largest logit in equal steps, then of the logit's own bits, then of the id's,
// until the bin that the border falls into has at most kList elements; those are compared one by one.  Weights are whole numbers (1, where elements are
// counted), so the order of the atomic additions does not matter.  What costs is additions of a wavefront to the same bin, some 50 cycles each: hence equal
// steps, as many as there is room for, and one addition where all lanes' logits are the same.
template <int W, int BITS, typename Weight = uint64_t> struct Search {
    uint64_t sum[1 << BITS];
    uint64_t part[W], before;
    Weight w[kList];
    float low[W];
    int bin;
    Place last;
};

// Before each search: the least logit of the order, and empty bins.  A barrier has to follow.
template <typename T, int BITS, int W, typename Weight, typename Source> __device__ __forceinline__ void begin_search(const Source& source, Search<W, BITS, Weight>& h) {
    constexpr int N = RowVec<T>::n;
    float low = kInf;
    source.logits([&](int, float (&z)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) low = fminf(low, z[e] > -kInf ? z[e] : kInf);
    });
    low = wave_min(low);
    if ((threadIdx.x & 63) == 0) h.low[threadIdx.x >> 6] = low;
    for (int i = threadIdx.x; i < 1 << BITS; i += 64 * W) h.sum[i] = 0;
}

// source.each(f): f(first id, logits, weights) for every vector of the row; what weighs 0 takes no part (minus infinity and NaN among it, and something has
// to take part); source.logits(f): f(first id, logits) for every vector; source.logit(id), source.weight(logit, id): of one element.  target_of(all): the least
// sum of weights that the part up to its last element reaches, of the sum of all; 0 is as good as 1, and what is more than there is counts as all.  span: what
// is further than that from the largest weighs 0, or nothing is known about it (infinity).
template <typename T, int BITS, int W, typename Weight, typename Source, typename F>
__device__ __forceinline__ Place find_last(const Source& source, float top, float span, F target_of, Search<W, BITS, Weight>& h, List& list) {
    constexpr int N = RowVec<T>::n, kThreads = 64 * W, kBins = 1 << BITS, kEach = kBins < kThreads ? 1 : kBins / kThreads, kIdBits = 18;
    static_assert(kMostVocab <= 1 << kIdBits, "an id's digits");
    constexpr int kZLevels = (32 + BITS - 1) / BITS, kLevels = 1 + kZLevels + (kIdBits + BITS - 1) / BITS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int bin0 = 0;
    uint32_t bits = 0, id_bits = 0;      // digits found so far
    int known = 32, id_known = kIdBits;  // and how many bits are below them
    uint64_t passed = 0, target = 0;     // passed: in front of the bin
    float low = h.low[0];
#pragma unroll
    for (int i = 1; i < W; ++i) low = fminf(low, h.low[i]);
    const float rate = (float)kBins / fminf(fmaxf(top - low, 0x1p-100f), span);
    auto bin_of = [&](float z) { return (int)fminf((top - z) * rate, (float)(kBins - 1)); };
    auto in_bin = [&](float z, int id) {
        if (known == 32) return bin_of(z) == bin0;
        return bin_of(z) == bin0 && (uint64_t)(~rising_bits(z) ^ bits) >> known == 0 && ((uint32_t)id ^ id_bits) >> id_known == 0;
    };
    for (int level = 0;; ++level) {
        const bool by_z = level <= kZLevels;
        const int have = by_z ? known : id_known, take = min(BITS, have), shift = have - take;
        if (level == 0) {
            source.each([&](int, const float (&z)[N], const uint64_t (&w)[N]) {
                const float one = bits_f32(__builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, z[0])));
                bool alike = z[0] == one;  // the whole wavefront's logits are one
                if (__all(alike)) {
#pragma unroll
                    for (int e = 0; e < N; ++e) alike = alike && w[e] != 0 && z[e] == one;
                }
                if (__all(alike)) {
                    if (lane == 0) atomicAdd((unsigned long long*)&h.sum[bin_of(one)], (unsigned long long)(w[0] * (64 * N)));
                    return;
                }
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (w[e] != 0) atomicAdd((unsigned long long*)&h.sum[bin_of(z[e])], (unsigned long long)w[e]);
            });
        } else {
            source.each([&](int first, const float (&z)[N], const uint64_t (&w)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int id = first + e;
                    const bool counts = w[e] != 0 && in_bin(z[e], id);
                    const int digit = ((by_z ? ~rising_bits(z[e]) : (uint32_t)id) >> shift) & ((1u << take) - 1);
                    const uint64_t lanes = __ballot(counts);
                    if (lanes == 0) continue;
                    const int one = __builtin_ctzll(lanes);
                    if (by_z && __ballot(counts && z[e] == bits_f32(lane_of(__builtin_bit_cast(uint32_t, z[e]), one))) == lanes) {
                        if (lane == one) atomicAdd((unsigned long long*)&h.sum[digit], (unsigned long long)(w[e] * __builtin_popcountll(lanes)));
                    } else if (counts) {
                        atomicAdd((unsigned long long*)&h.sum[digit], (unsigned long long)w[e]);
                    }
                }
            });
        }
        __syncthreads();
        uint64_t mine = 0;
        if (tid < kBins)
            for (int i = 0; i < kEach; ++i) mine += h.sum[kEach * tid + i];
        const uint64_t through = wave_prefix(mine);
        if (lane == 63) h.part[wave] = through;
        if (tid == 0) list.count = 0;
        __syncthreads();
        uint64_t at = passed + through - mine, all = passed;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            at += i < wave ? h.part[i] : 0;
            all += h.part[i];
        }
        if (level == 0) target = max(min(target_of(all), all), (uint64_t)1);  // there may be fewer
        if (at < target && target <= at + mine)
            for (int i = 0; i < kEach; ++i) {
                const uint64_t v = h.sum[kEach * tid + i];
                if (at < target && target <= at + v) {  // one bin of one thread
                    h.bin = kEach * tid + i;
                    h.before = at;
                }
                at += v;
            }
        __syncthreads();
        passed = h.before;
        if (level == 0) {
            bin0 = h.bin;
        } else if (by_z) {
            bits |= (uint32_t)h.bin << shift;
            known = shift;
        } else {
            id_bits |= (uint32_t)h.bin << shift;
            id_known = shift;
        }
        if (known == 32 && bin0 < kBins - 1) {  // of the distance in steps less the bin: 0 to 1 by its bits, so NaN and infinity are not in it
            const float bin = (float)bin0;
            source.logits([&](int id, float (&z)[N]) {
#pragma clang fp contract(off)  // the same product as bin_of's
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint32_t u = __builtin_bit_cast(uint32_t, (top - z[e]) * rate - bin);
                    z[e] = bits_f32(u | ~(u - 0x3f800000u));
                }
                put_in(list, id, z);
            });
        } else {
            source.logits([&](int id, float (&z)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e) z[e] = z[e] > -kInf && in_bin(z[e], id + e) ? 0.f : -1.f;
                put_in(list, id, z);
            });
        }
        __syncthreads();
        if (list.count <= kList || level + 1 == kLevels) break;
        for (int i = tid; i < kBins; i += kThreads) h.sum[i] = 0;
        __syncthreads();  // and all have read the count
    }
    const int n = min((int)list.count, kList);
    for (int i = tid; i < n; i += kThreads) {
        const int id = list.id[i];
        const float z = source.logit(id);
        list.key[i] = order_key(z, id);
        h.w[i] = (Weight)source.weight(z, id);
    }
    __syncthreads();
    if constexpr (kThreads > kList) {  // several neighbours for each element
        constexpr int kShare = kThreads / kList;
        static_assert(kShare <= 4, "within a quad");
        const int i = tid / kShare;
        if (i < n) {
            const uint64_t key = list.key[i], own = h.w[i];
            uint64_t at = 0;
#pragma unroll 8
            for (int j = tid % kShare; j < n; j += kShare) at += list.key[j] > key ? (uint64_t)h.w[j] : 0;
            at += dpp_mov64<0xB1>(at);
            if constexpr (kShare == 4) at += dpp_mov64<0x4E>(at);
            at += passed;
            if (at < target && target <= at + own) h.last = Place{key_logit(key), key_id(key)};
        }
    } else {
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t key = list.key[i], own = h.w[i];
            uint64_t at = passed;
#pragma unroll 8
            for (int j = 0; j < n; ++j) at += list.key[j] > key ? (uint64_t)h.w[j] : 0;
            if (at < target && target <= at + own) h.last = Place{key_logit(key), key_id(key)};
        }
    }
    __syncthreads();
    return h.last;
}

}  // namespace aed
