// The next token of a row of logits, by temperature, top-k, top-p and min-p, from a given random number.
//
//   w_i = exp((z_i - max) / t) over what the filters leave (each keeps a first part of the order); the token is the first id whose
//   sum of w up to it is above u times the whole sum
//
// A token is a border that a random number falls behind, and a filter's end another, so what matters is where sums lie, not how near they are: exponentials
// are taken in 64 bits and rounded to whole multiples of a power of two, whose sums are exact in any order.  With float32 sums one token in some
// thousands (a flat row of 4096) would be its neighbour.
//
// One workgroup a row.  Three ways through it, by what the row's own parameters ask for:
//   list    the filters leave few: those at or above a bound from the lanes' maxima are gathered in LDS and compared with each other
//   search  they leave many: the end of the first part is searched for by histograms (find_last)
//   sums    whatever is left is added up by runs of one wavefront's vector (256 or 512 ids in a row); the run that the random number falls into is
//           then gone through by one wavefront
#include "vocab_rows.h"

namespace aed {

namespace {

constexpr int kWanted = 64;      // gathered without top-k: a nucleus of a trained model's row is seldom larger
constexpr int kMostListed = 128;  // top-k above it goes by search

template <int W, int RUNS> struct SampleLds {
    RowBounds<W> bounds;
    List list;
    Search<W, 11, true> search;
    uint64_t w[kList];  // by id
    int by_place[kList], by_id[kList];
    float z[kList];
    uint64_t run[RUNS];
};

// 2^y, y <= 0, to some 2^-50: the exponential's series for the fraction, |y| <= 1/2: the term that is left out, (ln 2 / 2)^12 / 12!, is 6e-15.
__device__ __forceinline__ double pow2(double y) {
    y = fmax(y, -1100.0);
    const double n = rint(y), f = y - n;
    constexpr double l = 0.69314718055994530942;
    constexpr double c2 = l * l / 2, c3 = c2 * l / 3, c4 = c3 * l / 4, c5 = c4 * l / 5, c6 = c5 * l / 6, c7 = c6 * l / 7, c8 = c7 * l / 8, c9 = c8 * l / 9, c10 = c9 * l / 10,
                     c11 = c10 * l / 11;
    double p = fma(f, c11, c10);
    p = fma(f, p, c9);
    p = fma(f, p, c8);
    p = fma(f, p, c7);
    p = fma(f, p, c6);
    p = fma(f, p, c5);
    p = fma(f, p, c4);
    p = fma(f, p, c3);
    p = fma(f, p, c2);
    p = fma(f, p, l);
    p = fma(f, p, 1.0);
    return ldexp(p, (int)n);
}
struct Weigh {
    double top, c, magic;  // log2 e / t; 2^(52 - bits): a double there has whole multiples of 2^-bits as its last digits
    float top_f;
    __device__ __forceinline__ double exact(float z) const {
#pragma clang fp contract(off)  // the same weight wherever it is made
        const double w = z > -kInf && top_f < kInf ? pow2(((double)z - top) * c) : 0.0;
        return z == top_f ? 1.0 : w;
    }
    __device__ __forceinline__ uint64_t whole(double w) const {
#pragma clang fp contract(off)
        return __builtin_bit_cast(uint64_t, magic + w) - __builtin_bit_cast(uint64_t, magic);
    }
};

// floor(f n) or (UP) its ceiling, exactly; f in [0, 1]
template <bool UP> __device__ __forceinline__ uint64_t part_of(float f, uint64_t n) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, f), field = bits >> 23;
    const uint64_t digits = field ? (bits & 0x7fffffu) | 0x800000u : bits;
    const int down = 150 - max((int)field, 1);  // f = digits / 2^down, 23 to 149
    const uint64_t lo = digits * n, hi = __umul64hi(digits, n);
    uint64_t whole, left;
    if (down < 64) {
        whole = hi << (64 - down) | lo >> down;
        left = lo << (64 - down);
    } else {
        whole = down < 128 ? hi >> (down - 64) : 0;
        left = whole == 0 ? hi | lo : lo | (hi - (whole << (down - 64)));
    }
    return whole + (UP && left != 0);
}

template <int W> __device__ __forceinline__ uint64_t block_sum64(uint64_t v, uint64_t* part) {
    v = wave_sum64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v += part[i];
    return v;
}

}  // namespace

template <typename T, int W, int S, int RUNS> __global__ __launch_bounds__(64 * W) void sample_kernel(SampleArgs a) {
    constexpr int N = RowVec<T>::n;
    static_assert(64 * W >= kList && RUNS >= W, "a thread for each that is listed, sums of wavefronts in the runs' place");
    __shared__ SampleLds<W, RUNS> lds;
    List& list = lds.list;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Row<T, W, S> row(a.z, r);
    const float t = a.temperatures ? a.temperatures[r] : a.temperature;
    const bool greedy = !(t > 0.f);
    int k = a.top_ks ? a.top_ks[r] : a.top_k;
    k = greedy ? 1 : k <= 0 || k > a.z.vocab ? a.z.vocab : k;
    const float given_p = greedy ? 1.f : a.top_ps ? a.top_ps[r] : a.top_p, top_p = fmaxf(given_p, 0.f), min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const bool by_k = k < a.z.vocab, by_p = given_p < 1.f;  // not by NaN
    const double least = greedy || !(min_p > 0.f) ? 0.0 : (double)fminf(min_p, 1.f);
    const float u0 = a.uniforms[r];
    const float u = u0 > 0.f ? fminf(u0, 1.f) : 0.f;

    float top, bound;
    bound_row<W>(row, by_k ? (k <= kMostListed ? k : 1) : by_p ? kWanted : 1, lds.bounds, list, top, bound);
    row.forget();
    if (!(top > -kInf)) {  // nothing to draw from
        if (tid == 0) {
            a.tokens[r] = -1;
            a.logp[r] = -kInf;
        }
        return;
    }
    Weigh weigh;
    weigh.top_f = top;
    weigh.top = top;
    weigh.c = greedy ? 0.0 : kLog2eD / (double)t;
    weigh.magic = __builtin_bit_cast(double, (uint64_t)(1023 + 52 - a.weight_bits) << 52);
    auto weight = [&](float z) { return weigh.whole(weigh.exact(z)); };
    // runs' sums of what `in` leaves and min-p does
    auto add_runs = [&](auto in) {
        row.each_vec([&](int s, int id, const auto& v) {
            uint64_t mine = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float z = to_f32((T)v[e]);
                if (in(z, id + e)) {
                    const double w = weigh.exact(z);
                    mine += w >= least ? weigh.whole(w) : 0;
                }
            }
            mine = wave_sum64(mine);
            if (lane == 0) lds.run[s * W + wave] = mine;
        });
    };
    auto anything = [](float, int) { return true; };
    const int runs = ((a.z.vocab + N - 1) / N + 63) / 64;

    Place last{-kInf, INT_MAX};  // of A, then of B
    if (by_k || by_p) {
        bool few = !by_k || k <= kMostListed;
        uint64_t all = 0;  // A's sum, if A is the whole row
        if (few) {
            uint64_t mine = 0;
            gather(row, bound, list, [&](float z, float) {
                if (!by_k) mine += weight(z);
            });
            if (!by_k) all = block_sum64<W>(mine, lds.run);
        }
        const int n = few ? (int)list.count : 0;
        few = few && n <= kList;
        if (few) {
            // each by its thread: its place in the order, and among the ids
            if (tid < n) list.z[tid] = in_order(to_f32(row.p[list.id[tid]]));
            __syncthreads();
            if (tid < n) {
                const float z = list.z[tid];
                const int id = list.id[tid];
                int place = 0, by_id = 0;
#pragma unroll 8
                for (int j = 0; j < n; ++j) {
                    place += before(list.z[j], list.id[j], z, id);
                    by_id += list.id[j] < id;
                }
                lds.z[place] = z;
                lds.by_place[place] = by_id;
                lds.by_id[by_id] = id;
            }
            __syncthreads();
            // in their order, four a lane, by the first wavefront
            constexpr int kEach = kList / 64;
            uint64_t w[kEach], mine = 0, of_a = 0;
            double x[kEach];
            if (wave == 0) {
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int place = kEach * lane + i;
                    x[i] = place < n ? weigh.exact(lds.z[place]) : 0.0;
                    w[i] = place < n ? weigh.whole(x[i]) : 0;
                    mine += w[i];
                    of_a += place < k ? w[i] : 0;
                }
                of_a = wave_sum64(of_a);  // A's sum, or that of its listed part
            }
            bool found = by_k;
            if (!by_k) {
                if (tid == 0) lds.run[0] = of_a;
                __syncthreads();
                of_a = lds.run[0];
                found = of_a >= part_of<true>(top_p, all);  // all of B is listed
            }
            if (found) {
                if (wave != 0) return;
                const uint64_t border = by_p ? part_of<true>(top_p, by_k ? of_a : all) : ~(uint64_t)0;
                uint64_t front = wave_prefix(mine) - mine, left = 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int place = kEach * lane + i;
                    const uint64_t kept = place < k && (place == 0 || front < border) && x[i] >= least ? w[i] : 0;
                    front += w[i];
                    left += kept;
                    if (place < n) lds.w[lds.by_place[place]] = kept;
                }
                left = wave_sum64(left);
                other_lanes_wrote();
                const uint64_t target = min(part_of<false>(u, left), left - 1);
                uint64_t v[kEach];
                mine = 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) mine += v[i] = kEach * lane + i < n ? lds.w[kEach * lane + i] : 0;
                uint64_t at = wave_prefix(mine) - mine;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    if (at <= target && target < at + v[i]) {
                        a.tokens[r] = lds.by_id[kEach * lane + i];
                        a.logp[r] = (float)log((double)v[i] / (double)left);
                    }
                    at += v[i];
                }
                return;
            }
        }
        __syncthreads();
        if (by_k) last = find_last<false>(row.again(), top, k, lds.search, list, anything, weight);
        if (by_p) {
            if (by_k) {
                uint64_t mine = 0;
                row.each([&](float z, int id) {
                    if (up_to(z, id, last)) mine += weight(z);
                });
                all = block_sum64<W>(mine, lds.run);
            }
            const uint64_t border = max(part_of<true>(top_p, all), (uint64_t)1);
            const Place of_a = last;
            last = find_last<true>(row.again(), top, border, lds.search, list, [=](float z, int id) { return up_to(z, id, of_a); }, weight);
        }
    }
    add_runs([=](float z, int id) { return up_to(z, id, last); });
    __syncthreads();
    if (wave != 0) return;
    uint64_t left = 0;
    for (int i = lane; i < runs; i += 64) left += lds.run[i];
    left = wave_sum64(left);
    const uint64_t target = min(part_of<false>(u, left), left - 1);
    uint64_t at = 0;  // in front of the runs that are looked at
    int found = -1;
    for (int first = 0; found < 0 && first < runs; first += 64) {
        const uint64_t v = first + lane < runs ? lds.run[first + lane] : 0, through = at + wave_prefix(v);
        const uint64_t hit = __ballot(through > target);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            found = first + l;
            at = lane_of(through - v, l);
        } else {
            at = lane_of(through, 63);
        }
    }
    // the run's ids, N a lane
    const int id0 = (found * 64 + lane) * N, id = vec_begin<N>(id0, a.z.vocab);
    const auto v = row_vec(row.p, id0, a.z.vocab);
    uint64_t w[N], mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float z = to_f32((T)v[e]);
        const double x = z > -kInf && up_to(z, id + e, last) ? weigh.exact(z) : 0.0;
        w[e] = x > 0.0 && x >= least ? weigh.whole(x) : 0;
        mine += w[e];
    }
    at += wave_prefix(mine) - mine;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (at <= target && target < at + w[e]) {
            a.tokens[r] = id + e;
            a.logp[r] = (float)log((double)w[e] / (double)left);
        }
        at += w[e];
    }
}

namespace {

template <typename T, int W, int S> hipError_t launch_sample_as(const SampleArgs& a, hipStream_t s) {
    constexpr int runs = S > 0 ? S * W : kMostVocab / (64 * RowVec<T>::n);
    sample_kernel<T, W, S, runs><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t launch_sample_of(const SampleArgs& a, hipStream_t s) {
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    if (vecs <= 256 * 4) return launch_sample_as<T, 4, 4>(a, s);
    if (vecs <= 1024 * 8) return launch_sample_as<T, 16, 8>(a, s);
    return launch_sample_as<T, 16, 0>(a, s);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t s) { return bf16 ? launch_sample_of<bf16_t>(a, s) : launch_sample_of<float>(a, s); }

}  // namespace aed
