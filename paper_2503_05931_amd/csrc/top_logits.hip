// A row's largest logits, in order, with their ids, and the log of the sum of exponentials of all others.
//
// Bound by memory: a row is read once, into registers.  Its lanes' maxima give a bound that a few more elements than are asked for are not below; those are
// gathered in LDS and placed by comparing each with each.  Everything below the bound adds to the rest's sum in the same pass, relative to the
// bound, so nothing is subtracted from a whole row's sum, however little is left of it.  32 of 4096 in bfloat16, 8448 rows: 18.9 us, 3.8 TB/s with a launch's 4 us;
// 64 of 32768, 2048 rows: 33 us, 4.1 TB/s.  With 128 asked for comparisons count: 44 us for the former.
#include "vocab_rows.h"

namespace aed {

namespace {

constexpr float kLn2 = 0.69314718055994530942f;

template <int W> struct TopLds {
    RowBounds<W> bounds;
    List list;
    Search<W, 8, uint8_t> search;
    float part[W];
    float over[kList];
    uint32_t place[W > 1 ? kList : 1];
};
// Each one's place: put(key, how many of the n keys are larger).  A lane has M of them, so that a key that is read from LDS, where all lanes take the same, is
// compared M times: reading costs more than comparing.  Wavefronts share the keys to compare with.  64 of 4096 in bfloat16, 8448 rows: 25.9 us, and 28.2 with one key
// a lane at a time.
template <int W, int M, typename F> __device__ __forceinline__ void place_all(TopLds<W>& lds, int n, F put) {
    if (n == 0) return;  // there is no key to read
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t key[M];
    uint32_t place[M] = {};
#pragma unroll
    for (int i = 0; i < M; ++i) key[i] = lds.list.key[min(64 * i + lane, n - 1)];
#pragma unroll 8
    for (int j = wave; j < n; j += W) {
        const uint64_t other = lds.list.key[j];
#pragma unroll
        for (int i = 0; i < M; ++i) place[i] += other > key[i];
    }
    if constexpr (W == 1) {
#pragma unroll
        for (int i = 0; i < M; ++i)
            if (64 * i + lane < n) put(key[i], place[i]);
    } else {
#pragma unroll
        for (int i = 0; i < M; ++i)
            if (64 * i + lane < n) atomicAdd(&lds.place[64 * i + lane], place[i]);
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += 64 * W) put(lds.list.key[i], lds.place[i]);
    }
}
// every element of the order counts 1
template <typename T, int W> struct Counted {
    static constexpr int N = RowVec<T>::n;
    RowLoop<T, W> loop;
    template <typename F> __device__ __forceinline__ void logits(F f) const {
        loop.each_floats([&](int, int id, float (&z)[N]) { f(id, z); });
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
        loop.each_floats([&](int, int id, float (&z)[N]) {
            uint64_t w[N];
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = z[e] > -kInf;
            f(id, z, w);
        });
    }
    __device__ __forceinline__ float logit(int id) const { return to_f32(loop.p[id]); }
    __device__ __forceinline__ uint64_t weight(float z, int) const { return z > -kInf; }
};
template <int W> __device__ __forceinline__ float block_sum(float v, float* part) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        __syncthreads();  // part is free
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int i = 1; i < W; ++i) v += part[i];
    }
    return v;
}
template <int W> __device__ __forceinline__ float block_max(float v, float* part) {
    v = wave_max(v);
    if constexpr (W > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int i = 1; i < W; ++i) v = fmaxf(v, part[i]);
    }
    return v;
}

}  // namespace

template <typename T, int W, int S> __global__ __launch_bounds__(64 * W) void top_logits_kernel(TopArgs a) {
    constexpr int kThreads = 64 * W;
    __shared__ TopLds<W> lds;
    List& list = lds.list;
    const int r = blockIdx.x, tid = threadIdx.x, K = a.top;
    Row<T, W, S> row(a.z, r);
    float* const values = a.values + (int64_t)r * K;
    int32_t* const ids = a.ids + (int64_t)r * K;
    float top, bound;
    bound_row<W>(row, K, lds.bounds, list, top, bound);
    row.forget();
    const RowLoop<T, W> loop{row.p, row.n};
    float border, sum;  // sum: of what is below the border, relative to it; may be NaN, if one is in the row
    bool fits;
    auto take = [&](const auto& from) {
        // Exponents relative to a border that the bound's own product, rounded, is not below.  Where a product could be infinite, the row is searched; where the
        // sum is (what is listed may lie far above the border, if that is large), it is made again below.
        // The border is never within 2^-41 of 0.  So what is below it is by 2^-89 at least (a product of two floats at 2^-42 is a multiple of that, the
        // border of 2^-65), and counts whole: 2^100 times as much is above 1.  What lies around 0 is listed then; a row that has nothing else is searched.
        bound = gather_bound(bound);
        const float scaled = bound * a.scale;
        border = fabsf(scaled) >= 0x1p-40f ? scaled - fabsf(scaled) * 0x1p-22f : -0x1p-39f;
        fits = fabsf(scaled) < 1e37f;
        sum = 0.f;
        gather(from, list, [&](float (&z)[RowVec<T>::n]) {
#pragma unroll
            for (int e = 0; e < RowVec<T>::n; ++e) {
                z[e] = fmaf(z[e], a.scale, -border);
                const float below = __builtin_amdgcn_fmed3f(z[e] * -0x1p100f, 0.f, 1.f);
                sum = fmaf(__builtin_amdgcn_exp2f(z[e]), below, sum);
            }
        });
        asm volatile("" : "+v"(sum));  // it is made here, not where it is used: there the row would have to be kept
    };
    take(row);
    const bool again = list.count > kList;
    if (again) {
        bound = listed_bound<W>(row.p, list, K);
        take(Row<T, W, 0>(row.p, row.n));
    }
    int n = list.count;
    Place last{-kInf, INT_MAX};
    const bool searched = n > kList || !fits;
    if (searched) {  // many equal ones, mostly
        if (top > -kInf) {
            const Counted<T, W> source{loop};
            begin_search<T>(source, lds.search);
            __syncthreads();
            last = find_last<T>(source, top, kInf, [&](uint64_t) { return (uint64_t)K; }, lds.search, list);
        }
        __syncthreads();  // every wavefront has come here by the count
        if (tid == 0) list.count = 0;
        __syncthreads();
        loop.each_floats([&](int, int id, float (&z)[RowVec<T>::n]) {
#pragma unroll
            for (int e = 0; e < RowVec<T>::n; ++e) z[e] = z[e] > -kInf && up_to(z[e], id + e, last) ? 0.f : -1.f;
            put_in(list, id, z);
        });
        __syncthreads();
        n = list.count;
    }
    read_keys<W>(row.p, list, n);
    if constexpr (W > 1)
        for (int i = tid; i < kList; i += kThreads) lds.place[i] = 0;
    __syncthreads();
    auto put = [&](uint64_t key, int place) {
        const float z = key_logit(key);
        if (place < K) {
            values[place] = z;
            ids[place] = z > -kInf ? key_id(key) : -1;
            if (place == K - 1) lds.search.last = Place{z, key_id(key)};
        } else {
            lds.over[place] = z;
        }
    };
    if (n <= 64) place_all<W, 1>(lds, n, put);
    else if (n <= 128) place_all<W, 2>(lds, n, put);
    else place_all<W, 4>(lds, n, put);
    for (int i = n + tid; i < K; i += kThreads) {
        values[i] = -kInf;
        ids[i] = -1;
    }
    float rest = -kInf;
    if (n >= K) {  // there may be others
        __syncthreads();
        // listed, but not among the first: in their order, as the list has none
        for (int i = K + tid; i < n; i += kThreads) sum += __builtin_amdgcn_exp2f(fmaf(lds.over[i], a.scale, -border));
        sum = searched || (again && W > 1) ? 0.f : block_sum<W>(sum, lds.part);  // the second bound is that of what was listed first, by whichever wavefront
        if (sum >= 0x1p-60f && sum < 0x1p100f) {
            rest = kLn2 * (border + __builtin_amdgcn_logf(sum));
        } else {  // nothing, or far from the border, or by another one each time: relative to its own largest
            last = lds.search.last;
            float m = -kInf;
            loop.each([&](float z, int id) { m = up_to(z, id, last) ? m : fmaxf(m, z); });
            const float base = block_max<W>(m, lds.part);
            sum = 0.f;
            if (base > -kInf) loop.each([&](float z, int id) { sum += z > -kInf && !up_to(z, id, last) ? __builtin_amdgcn_exp2f((z - base) * a.scale) : 0.f; });
            sum = block_sum<W>(sum, lds.part);
            if (base > -kInf) rest = base == kInf ? kInf : base / a.temperature + logf(sum);
        }
    }
    if (tid == 0) a.rest[r] = rest;
}

namespace {

template <typename T, int W, int S> hipError_t launch_top_as(const TopArgs& a, hipStream_t s) {
    top_logits_kernel<T, W, S><<<dim3(a.z.rows), dim3(64 * W), 0, s>>>(a);
    return hipGetLastError();
}
// One wavefront has no barriers to wait at and lists the fewest elements; more are for what one has no registers for.  8448 rows of 4096 in bfloat16, 32 of them:
// one 18.2 us, four 31.2, 128 of them 44.8 and 54.2; 2048 of 32768, 64 of them: four 35.4, sixteen 92; 2048 of 65536: eight 84, sixteen 120.  Rows that no registers hold, 256 of 262144 in
// float32: eight wavefronts 96, sixteen 212; 4 of 131072: 31 and 22.
constexpr int kManyRows = 256;

template <typename T> hipError_t launch_top_of(const TopArgs& a, hipStream_t s) {
    const int vecs = (a.z.vocab + RowVec<T>::n - 1) / RowVec<T>::n;
    if (vecs <= 64 * 2) return launch_top_as<T, 1, 2>(a, s);
    if (vecs <= 64 * 8) return launch_top_as<T, 1, 8>(a, s);
    if (vecs <= 256 * 4) return launch_top_as<T, 4, 4>(a, s);
    if (vecs <= 256 * 16) return launch_top_as<T, 4, 16>(a, s);
    if (vecs <= 512 * 16) return launch_top_as<T, 8, 16>(a, s);
    return a.z.rows >= kManyRows ? launch_top_as<T, 8, 0>(a, s) : launch_top_as<T, 16, 0>(a, s);
}

}  // namespace

hipError_t launch_top(const TopArgs& a, bool bf16, hipStream_t s) { return bf16 ? launch_top_of<bf16_t>(a, s) : launch_top_of<float>(a, s); }

}  // namespace aed
