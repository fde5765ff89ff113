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
//   list    the filters leave few: those at or above a bound (from the lanes' maxima, or min-p's) are gathered in LDS and compared with each other
//   search  they leave many: the end of the first part is searched for by histograms (find_last)
//   sums    whatever is left is added up by runs of one wavefront's vector (256 or 512 ids in a row); the run that the random number falls into is
//           then gone through by one wavefront
//
// Bound by latency in small calls (1 row of 4096: 4.5 us without filters, 6.2 by top-k 50, 9.7 by top-p 0.9, of which 4 are a launch and its first
// access; a search goes through some ten barriers, and what lies between them is a hundred or two of instructions of eight wavefronts that wait for each other) and by
// vector instructions in large ones: some 22 a weight, made once without filters (1024 rows of 4096 in float32: 9.1 us), twice in a search, once for the
// histogram and once for the runs (128 of 32768 in bfloat16 by top-p: 40 us; histogram 11, runs 10, whether a list will do 4, the row's bound, its least logit and
// the border's bin 9; half of the compute units have no row).
#include "vocab_rows.h"

namespace aed {

namespace {

constexpr int kWanted = 64;  // gathered for top-p: a nucleus of a trained model's row is seldom larger
// Rows of up to 4096, two a compute unit, have eight wavefronts each, whose threads hold their weights in registers.  Of 4096 in float32, by top-p: 256 rows with
// eight 10.7 us, with four 16.5; 512 rows 15.9 and 19.2; 1024 rows 28.9 and 25.1, by top-k 15.4 and 9.7, without filters 11.4 and 9.2.
constexpr int kFewRows = 512;
constexpr int kMostListed = 128;  // top-k above it goes by search: half a list, as the bound lets more in than are asked for

template <int W, int RUNS> struct SampleLds {
    static constexpr int kBits = W > 4 ? 11 : 10;
    RowBounds<W> bounds;
    List list;
    Search<W, kBits> search;
    uint64_t w[kList];    // by id
    uint64_t key[kList];  // by place
    int by_place[kList];
    uint64_t by_id[kList];  // keys
    uint64_t run[RUNS];
    float2 estimate[W];
};

// Weights of a row's logits
struct Weigh {
    Pow2 pow2;
    double top, c;  // c: log2 e / t
    double magic;   // 2^(52 - bits): a double there has whole multiples of 2^-bits as its last digits, and its own last 32 bits are 0
    float top_f;
    __device__ __forceinline__ Weigh(float top, float t, int bits)
        : top(top), c(t > 0.f ? kLog2eD / (double)t : 0.0), magic(__builtin_bit_cast(double, (uint64_t)(1023 + 52 - bits) << 52)), top_f(top) {}
    // exactly 1 for the largest; 0 for minus infinity and NaN, and for all but the largest where that is infinite
    template <int N> __device__ __forceinline__ void exact(const float (&z)[N], double (&x)[N]) const {
#pragma clang fp contract(off)  // the same weight wherever it is made
        constexpr int M = N < 4 ? N : 4;  // as many at once as the registers are for
#pragma unroll
        for (int first = 0; first < N; first += M) {
            double y[M];
#pragma unroll
            for (int e = 0; e < M; ++e) y[e] = ((double)z[first + e] - top) * c;
            pow2(y);
#pragma unroll
            for (int e = 0; e < M; ++e) x[first + e] = z[first + e] == top_f ? 1.0 : y[e];
        }
    }
    __device__ __forceinline__ double exact(float z) const {
        const float one[1] = {z};
        double x[1];
        exact(one, x);
        return x[0];
    }
    template <int N> __device__ __forceinline__ void wholes(const float (&z)[N], uint64_t (&w)[N]) const {
        double x[N];
        exact(z, x);
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = whole(x[e]);
    }
    __device__ __forceinline__ uint64_t whole(double w) const {
#pragma clang fp contract(off)
        const uint64_t u = __builtin_bit_cast(uint64_t, magic + w);
        return (uint64_t)((uint32_t)(u >> 32) - (uint32_t)(__builtin_bit_cast(uint64_t, magic) >> 32)) << 32 | (uint32_t)u;
    }
};

// log(weight of z / all), of which `part` whole multiples are counted, 0 < part <= all; bits: what they are multiples of.  From the logit itself: of a weight of
// 2^-40 its multiples of 2^-50 have three digits.
__device__ __forceinline__ float log_ratio(const Weigh& weigh, float z, uint64_t part, uint64_t all, int bits) {
    const double of_z = z == weigh.top_f ? 0.0 : ((double)z - weigh.top) * weigh.c;
    return part == all ? 0.f : (float)((of_z - log2_of(weigh.pow2, ldexp((double)all, -bits))) * (1 / kLog2eD));
}

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

// the workgroup's sums of two; part: 2 W
template <int W> __device__ __forceinline__ void block_sum64(uint64_t& a, uint64_t& b, uint64_t* part) {
    a = wave_sum64(a);
    b = wave_sum64(b);
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = a;
        part[W + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = part[0];
    b = part[W];
#pragma unroll
    for (int i = 1; i < W; ++i) {
        a += part[i];
        b += part[W + i];
    }
}
template <int W> __device__ __forceinline__ void block_sum32(float& a, float& b, float2* part) {
    a = (float)wave_sum((double)a);
    b = (float)wave_sum((double)b);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        a += part[i].x;
        b += part[i].y;
    }
}

// What find_last goes through: the elements up to `among`, that count 1 each or their weights.  Held: their weights (or 1, or 0) are in registers.
template <typename T, int W, int S> struct Held {
    static constexpr int N = RowVec<T>::n;
    const Row<T, W, S>& row;
    const uint64_t (&w)[S][N];
    const Weigh& weigh;
    Place among;
    bool by_weight;
    template <typename F> __device__ __forceinline__ void logits(F f) const {
        row.each_floats([&](int, int id, float (&z)[N]) {
            anew(z);
            f(id, z);
        });
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
        row.each_floats([&](int s, int id, float (&z)[N]) {
            anew(z);
            uint64_t v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[e] = w[s][e];
                asm volatile("" : "+v"(v[e]));
            }
            f(id, z, v);
        });
    }
    __device__ __forceinline__ float logit(int id) const { return to_f32(row.p[id]); }
    __device__ __forceinline__ uint64_t weight(float z, int id) const {
        return z > -kInf && up_to(z, id, among) ? by_weight ? weigh.whole(weigh.exact(z)) : 1 : 0;
    }
    // or what a pass makes of the logits is kept for the next one, and there are no registers for it
    static __device__ __forceinline__ void anew(float (&z)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) asm volatile("" : "+v"(z[e]));
    }
};
// Made: weights are made anew in each pass, from the row in memory.
template <typename T, int W> struct Made {
    static constexpr int N = RowVec<T>::n;
    RowLoop<T, W> loop;
    const Weigh& weigh;
    Place among;
    bool by_weight;
    template <typename F> __device__ __forceinline__ void logits(F f) const {
        loop.each_floats([&](int, int id, float (&z)[N]) { f(id, z); });
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
        loop.each_floats([&](int, int id, float (&z)[N]) {
            uint64_t w[N];
            if (by_weight) weigh.wholes(z, w);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = takes_part(z[e], id + e) ? by_weight ? w[e] : 1 : 0;
            f(id, z, w);
        });
    }
    __device__ __forceinline__ float logit(int id) const { return to_f32(loop.p[id]); }
    __device__ __forceinline__ uint64_t weight(float z, int id) const { return takes_part(z, id) ? by_weight ? weigh.whole(weigh.exact(z)) : 1 : 0; }
    __device__ __forceinline__ bool takes_part(float z, int id) const { return z > -kInf && up_to(z, id, among); }
};

}  // namespace

template <typename T, int W, int S, int RUNS> __global__ __launch_bounds__(64 * W, 4) void sample_kernel(SampleArgs a) {
    constexpr int N = RowVec<T>::n;
    constexpr bool kHeld = S > 0 && S * N <= 8;  // a thread's weights have room in registers
    constexpr bool kKept = kHeld;  // the row too, to the end (1024 rows, four wavefronts each, without filters: 9.9 us, and 9.2 read anew by the first)
    static_assert(64 * W >= kList && RUNS >= 2 * W, "a thread for each that is listed, sums of wavefronts in the runs' place");
    typedef SampleLds<W, RUNS> Lds;
    __shared__ Lds lds;
    List& list = lds.list;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Row<T, W, S> row(a.z, r);
    const float t = a.temperatures ? a.temperatures[r] : a.temperature;
    const bool greedy = !(t > 0.f);
    int k = a.top_ks ? a.top_ks[r] : a.top_k;
    k = greedy ? 1 : k <= 0 || k > a.z.vocab ? a.z.vocab : k;
    const float given_p = greedy ? 1.f : a.top_ps ? a.top_ps[r] : a.top_p, top_p = fmaxf(given_p, 0.f), min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const bool by_k = k < a.z.vocab, by_p = given_p < 1.f;  // not by NaN
    const float least = greedy || !(min_p > 0.f) ? 0.f : fminf(min_p, 1.f);
    // the least weight that min-p leaves
    const uint64_t least_w = (uint64_t)ceil((double)least * __builtin_bit_cast(double, (uint64_t)(1023 + a.weight_bits) << 52));
    const float u0 = a.uniforms[r];
    const float u = u0 > 0.f ? fminf(u0, 1.f) : 0.f;

    float top, bound;
    bound_row<W>(row, by_k ? (k <= kMostListed ? k : 0) : by_p ? kWanted : 0, lds.bounds, list, top, bound);
    row.forget();
    if (!(top > -kInf)) {  // nothing to draw from
        if (tid == 0) {
            a.tokens[r] = -1;
            a.logp[r] = -kInf;
        }
        return;
    }
    const Weigh weigh(top, greedy ? 0.f : t, a.weight_bits);
    const RowLoop<T, W> loop{row.p, row.n};
    uint64_t held[kHeld ? S : 1][N];
    int token = -1;  // of the lane that finds it
    float its_z = 0.f;
    uint64_t its = 0, left = 0;

    Place last{-kInf, INT_MAX};  // of A, then of B
    const bool by_least = least > 0.f, needs_a = by_k && by_p;  // A's sum, from the list
    if (by_k || by_p || by_least) {
        uint64_t all = 0;  // A's sum
        float least_bound = -kInf;
        if (by_least && !needs_a) {  // what min-p takes out need not be listed; a little below its end, as that is rounded
            const float end = t * logf(least);
            least_bound = fmaxf(top + end - 1e-5f * (fabsf(top) + fabsf(end)), -kInf);
        }
        const bool complete = least_bound >= bound && weigh.whole(weigh.exact(least_bound)) < least_w;  // nothing below min-p's end is in C
        bound = gather_bound(fmaxf(bound, least_bound));
        bool few = complete || (by_k ? k <= kMostListed : by_p);
        // the whole row's sum, and whether all of B is at or above the bound
        auto whole_row = [&] {
            uint64_t mine = 0, above = 0;
            row.each_floats([&](int s, int, float (&z)[N]) {
                uint64_t w[N];
                weigh.wholes(z, w);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    mine += w[e];
                    above += z[e] - bound >= 0.f ? w[e] : 0;
                    if constexpr (kHeld) held[s][e] = w[e];
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            block_sum64<W>(mine, above, lds.run);
            all = mine;
            const bool within = above >= part_of<true>(top_p, all);
            row.forget();
            return within;
        };
        const bool of_row = by_p && !by_k;
        if (of_row) {
            if constexpr (kHeld) {
                few = whole_row() || complete;
            } else if (!complete) {  // by float32 whether it may be; a search needs no sum beforehand
                const float c = kLog2eD / t;
                float mine = 0.f, above = 0.f;
                row.each_floats([&](int, int, float (&z)[N]) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float x = fmaxf(__builtin_amdgcn_exp2f((z[e] - top) * c), 0.f);
                        mine += x;
                        above += z[e] - bound >= 0.f ? x : 0.f;
                    }
                });
                block_sum32<W>(mine, above, lds.estimate);
                few = !(above < 0.999f * top_p * mine);
                row.forget();
            }
        }
        bool known = !of_row || kHeld || complete;  // that what is needed is listed
        if (!few && least_bound > -kInf && weigh.whole(weigh.exact(least_bound)) < least_w) {  // perhaps min-p leaves few
            bound = gather_bound(least_bound);
            few = known = true;
        }
        if (few)
            gather(row, list, [&](float (&z)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e) z[e] -= bound;
            });
        if (few && by_k && k <= kMostListed && list.count > kList) {
            bound = gather_bound(listed_bound<W>(row.p, list, k));
            gather(Row<T, W, 0>(row.p, row.n), list, [&](float (&z)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e) z[e] -= bound;
            });
        }
        if constexpr (!kHeld)
            if (of_row && few && list.count <= kList) few = whole_row() || known;
        const int n = few ? (int)list.count : 0;
        if (few && n <= kList) {
            read_keys<W>(row.p, list, n);
            __syncthreads();
            {  // each one's place in the order, and among the ids, by neighbours that share the comparisons
                constexpr int kShare = 64 * W / kList;
                static_assert(kShare <= 4, "within a quad");
                const int i = tid / kShare;
                if (i < n) {
                    const uint64_t key = list.key[i];
                    uint32_t place = 0, by_id = 0;
#pragma unroll 8
                    for (int j = tid % kShare; j < n; j += kShare) {
                        place += list.key[j] > key;
                        by_id += (uint32_t)list.key[j] > (uint32_t)key;
                    }
                    uint64_t both = (uint64_t)by_id << 32 | place;
                    if constexpr (kShare > 1) both += dpp_mov64<0xB1>(both);
                    if constexpr (kShare > 2) both += dpp_mov64<0x4E>(both);
                    place = (uint32_t)both;
                    by_id = both >> 32;
                    if (tid % kShare == 0) {
                        lds.key[place] = key;
                        lds.by_place[place] = by_id;
                        lds.by_id[by_id] = key;
                    }
                }
            }
            __syncthreads();
            if (wave != 0) return;
            // in their order, by one wavefront
            constexpr int kEach = kList / 64;
            uint64_t w[kEach], of_a = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int place = 64 * i + lane;
                w[i] = 0;
                if (64 * i < n) w[i] = weigh.whole(weigh.exact(place < n ? key_logit(lds.key[place]) : -kInf));
                of_a += place < k ? w[i] : 0;
            }
            if (needs_a) all = wave_sum64(of_a);
            const uint64_t border = by_p ? part_of<true>(top_p, all) : 0;
            uint64_t front = 0;  // of the places that are looked at
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (64 * i >= n) continue;
                const int place = 64 * i + lane;
                const uint64_t through = front + wave_prefix(w[i]);
                const uint64_t kept = place < k && (place == 0 || !by_p || through - w[i] < border) && w[i] >= least_w ? w[i] : 0;
                front = lane_of(through, 63);
                left += kept;
                if (place < n) lds.w[lds.by_place[place]] = kept;
            }
            left = wave_sum64(left);
            other_lanes_wrote();
            const uint64_t target = min(part_of<false>(u, left), left - 1);
            uint64_t at = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (64 * i >= n) continue;
                const uint64_t v = 64 * i + lane < n ? lds.w[64 * i + lane] : 0, through = at + wave_prefix(v);
                if (through - v <= target && target < through) {
                    const uint64_t key = lds.by_id[64 * i + lane];
                    token = key_id(key);
                    its_z = key_logit(key);
                    its = v;
                }
                at = lane_of(through, 63);
            }
            if (token >= 0) {  // one lane
                a.tokens[r] = token;
                a.logp[r] = log_ratio(weigh, its_z, its, left, a.weight_bits);
            }
            return;
        }
        // the last of A by number, then that of B by weight
        auto search_in = [&](const auto& source, bool by_weight) {
            const float span = by_weight ? t * 45.f : kInf;  // a weight of e^-45 is nothing in units of 2^-50
            begin_search<T>(source, lds.search);
            __syncthreads();
            return find_last<T>(source, top, span, [&](uint64_t all) { return by_weight ? part_of<true>(top_p, all) : (uint64_t)k; }, lds.search, list);
        };
        auto search = [&](const Place& among, bool by_weight) {
            if constexpr (kHeld) return search_in(Held<T, W, S>{row, held, weigh, among, by_weight}, by_weight);
            else return search_in(Made<T, W>{loop, weigh, among, by_weight}, by_weight);
        };
#pragma unroll  // a search of each: what a loop shares has to be kept over it (64 rows by top-p: 10.3 us, and 10.8)
        for (int step = 0; step < 2; ++step) {
            const bool by_weight = step == 1;
            if (by_weight ? !by_p : !by_k) continue;
            if constexpr (kHeld) {
                if (by_k)  // 1 each, or those of A
                    row.each_floats([&](int s, int id, float (&z)[N]) {
                        uint64_t w[N];
                        Held<T, W, S>::anew(z);  // or the weights are made in front of the loop, for rows that need none too
                        if (by_weight) weigh.wholes(z, w);
#pragma unroll
                        for (int e = 0; e < N; ++e) held[s][e] = z[e] > -kInf && up_to(z[e], id + e, last) ? by_weight ? w[e] : 1 : 0;
                        __builtin_amdgcn_sched_barrier(0);
                    });
            }
            last = search(last, by_weight);
        }
    }
    // runs' sums of what is left
    const bool filtered = by_k || by_p || by_least;
    auto add_run = [&](int s, uint64_t mine) {
        mine = wave_sum64(mine);
        if (lane == 0) lds.run[s * W + wave] = mine;
        __builtin_amdgcn_sched_barrier(0);
    };
    if (filtered) {
        auto left_of = [&](int id, const float (&z)[N], const uint64_t (&w)[N]) {
            uint64_t mine = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) mine += up_to(z[e], id + e, last) && w[e] >= least_w ? w[e] : 0;
            return mine;
        };
        if (kHeld && by_p) {  // they are there
            if constexpr (kHeld) row.each_floats([&](int s, int id, float (&z)[N]) { add_run(s, left_of(id, z, held[s])); });
        } else {
            loop.each_floats([&](int s, int id, float (&z)[N]) {
                uint64_t w[N];
                weigh.wholes(z, w);
                add_run(s, left_of(id, z, w));
            });
        }
    } else {
        row.each_floats([&](int s, int, float (&z)[N]) {
            uint64_t w[N], mine = 0;
            weigh.wholes(z, w);
#pragma unroll
            for (int e = 0; e < N; ++e) mine += w[e];
            add_run(s, mine);
        });
    }
    __syncthreads();
    if (!kKept && wave != 0) return;
    const int runs = ((a.z.vocab + N - 1) / N + 63) / 64;
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
    typename RowVec<T>::type v;
    if constexpr (kKept) {  // by the wavefront that has it
        if (wave != found % W) return;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (s == found / W) v = row.x[s];
    } else {
        v = row_vec(row.p, id0, a.z.vocab);
    }
    float z[N];
    uint64_t w[N], mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = to_f32((T)v[e]);
    weigh.wholes(z, w);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        w[e] = up_to(z[e], id + e, last) && w[e] >= least_w ? w[e] : 0;
        mine += w[e];
    }
    at += wave_prefix(mine) - mine;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (at <= target && target < at + w[e]) {
            token = id + e;
            its_z = z[e];
            its = w[e];
        }
        at += w[e];
    }
    if (token >= 0) {  // one lane
        a.tokens[r] = token;
        a.logp[r] = log_ratio(weigh, its_z, its, left, a.weight_bits);
    }
}

namespace {

template <typename T, int W, int S> hipError_t launch_sample_as(const SampleArgs& a, hipStream_t s) {
    constexpr int runs = S > 0 ? S * W : kMostVocab / (64 * RowVec<T>::n);
    sample_kernel<T, W, S, (runs < 2 * W ? 2 * W : runs)><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    return hipGetLastError();
}
// Of 512 rows of 8000 in bfloat16 by top-p, eight wavefronts take 27 us, sixteen 44; of 256 of 14000 by top-k 50 8.5 and 21: sixteen fill a compute unit, and one row
// that is late leaves it idle.  Above 16384 sixteen have the registers: 128 of 32768 by top-p 40 us, eight 44.
template <typename T> hipError_t launch_sample_of(const SampleArgs& a, hipStream_t s) {
    constexpr int N = RowVec<T>::n;
    if (a.z.vocab <= 4096) return a.z.rows <= kFewRows ? launch_sample_as<T, 8, 8 / N>(a, s) : launch_sample_as<T, 4, 16 / N>(a, s);
    if (a.z.vocab <= 512 * 16) return launch_sample_as<T, 8, 16 / N>(a, s);
    if (a.z.vocab <= 512 * 32) return launch_sample_as<T, 8, 32 / N>(a, s);
    if (a.z.vocab <= 1024 * 32) return launch_sample_as<T, 16, 32 / N>(a, s);
    return launch_sample_as<T, 16, 0>(a, s);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t s) { return bf16 ? launch_sample_of<bf16_t>(a, s) : launch_sample_of<float>(a, s); }

}  // namespace aed
