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
    Histogram hist;
    uint64_t w[kList];
    uint64_t run[RUNS];
};

struct Weigh {
    double top, c, magic;  // log2 e / t; 2^(52 - bits): a double there has whole multiples of 2^-bits as its last digits
    float top_f;
    __device__ __forceinline__ double exact(float z) const {
#pragma clang fp contract(off)  // the same weight wherever it is made
        if (z == top_f) return 1.0;
        if (!(z > -kInf) || top_f == kInf) return 0.0;
        return exp2(((double)z - top) * c);
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
    const Row<T, W, S> row(a.z, r);
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
    auto gather = [&](float z, int id) {
        if (z >= bound && z > -kInf) put_in(list, z, id);
    };
    const int runs = ((a.z.vocab + N - 1) / N + 63) / 64;

    Place last{-kInf, INT_MAX};  // of A, then of B
    if (by_k || by_p) {
        bool listed = !by_k || k <= kMostListed;
        uint64_t all = 0;  // A's sum, if A is the whole row
        if (!by_k) {
            uint64_t mine = 0;
            row.each([&](float z, int id) {
                gather(z, id);
                mine += weight(z);
            });
            all = block_sum64<W>(mine, lds.run);
        } else if (listed) {
            row.each(gather);
        }
        __syncthreads();
        int n = list.count;
        listed = listed && n <= kList;
        if (listed) {
            // each by its thread: its weight, its place and what lies in front of it
            float z = -kInf;
            int id = -1, place = INT_MAX;
            uint64_t w = 0, front = 0;
            if (tid < n) {
                z = list.z[tid];
                id = list.id[tid];
                w = weight(z);
                lds.w[tid] = w;
            }
            __syncthreads();
            if (tid < n) {
                place = 0;
                for (int j = 0; j < n; ++j) {
                    const bool b = before(list.z[j], list.id[j], z, id);
                    place += b;
                    front += b ? lds.w[j] : 0;
                }
            }
            const uint64_t sum = block_sum64<W>(place < k ? w : 0, lds.run);  // of A, or of the part of it that is listed
            const uint64_t border = by_p ? part_of<true>(top_p, by_k ? sum : all) : ~(uint64_t)0;
            if (by_k || sum >= border) {  // all of B is listed
                const bool kept = place < k && (place == 0 || front < border) && weigh.exact(z) >= least;
                if (tid < n && !kept) lds.w[tid] = 0;
                const uint64_t left = block_sum64<W>(kept ? w : 0, lds.run);
                const uint64_t target = min(part_of<false>(u, left), left - 1);
                if (kept) {
                    uint64_t at = 0;
                    for (int j = 0; j < n; ++j) at += list.id[j] < id ? lds.w[j] : 0;
                    if (at <= target && target < at + w) {
                        a.tokens[r] = id;
                        a.logp[r] = (float)log((double)w / (double)left);
                    }
                }
                return;
            }
        }
        __syncthreads();
        if (by_k) last = find_last<false>(row.again(), top, k, lds.hist, list, anything, weight);
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
            last = find_last<true>(row.again(), top, border, lds.hist, list, [=](float z, int id) { return up_to(z, id, of_a); }, weight);
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
        const uint64_t v = first + lane < runs ? lds.run[first + lane] : 0, through = at + wave_prefix64(v);
        const uint64_t hit = __ballot(through > target);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            found = first + l;
            at = __shfl(through - v, l);
        } else {
            at = __shfl(through, 63);
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
    at += wave_prefix64(mine) - mine;
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
