// Attention of ragged batches, forward and backward: many rows a sequence against keys of another number, with an optional
// causal mask, byte mask of the keys and learned bias by the bucket of the distance.
//
//   s_ij = scale q_i . k_j + w[bucket(i, j)]   p = softmax of the visible   o_i = sum p v   lse_i = log sum exp s
//   dP = dO . V   delta_i = dO_i . O_i   dS = P (dP - delta)   dQ = scale dS K   dK = scale dS^T Q   dV = P^T dO
//   dw[b] = sum of dS over the pairs of bucket b
//
// Exponentials are powers of two: scores and bias carry log2 e.  Scores, softmax and sums are float32.  In bfloat16 the weights P and dS are
// rounded, where they become an operand of the second product: that product then runs at 16 times the float32 instructions' rate.  It costs
// as much as the rounding of the result itself does: outputs that are off by 0.0017 (2-norm, relative) from rounding alone are off by 0.0018 to
// 0.0020, dK and dV by 0.0024 (0.0017 in small batches, see there).  dQ's weights are rounded to 16 bits, a sum of two bfloat16, as it may have an error of delta besides (see there): 0.0017
// to 0.0018.  dw, sums of float32 dS, has its own rounding only.  No result depends on timing: whatever is added up has one
// order, and there are no atomics between wavefronts.
//
// Times in this file are the kernels' on an MI355X, bfloat16, 8 heads of 128, for the gradients' lists of four batches:
//   short  64 utterances, 4 909 rows (12 to 132), 9 021 keys           forward  19 us   dQ  28   dK and dV  33
//   long  128 utterances, 48 029 rows (300 to 448), 57 196 keys                189       280            384
//   self, short  64 sequences of 12 to 132 positions, causal, bias              15        32             28
//   self, long  128 sequences of 8 to 448 positions, causal, bias               72       176            144
// (those of the long batches move by 5 % and more with the card's clocks.)  The products of the long batch are 88, 132 and 176 GFLOP: 466, 471 and 458
// TFLOP/s, against 1 240 of a product of 8192 x 8192 x 8192; the second one of dQ's three, for the rest of dS, is not counted.
#include "attn_ragged.h"
#include "attn_tile.h"
#include "device_once.h"

#include <type_traits>

namespace aed {

namespace {

__device__ __forceinline__ float max_halves(float v) {
    const u32x2 a = swap32(v);
    return fmaxf(bits_f32(a[0]), bits_f32(a[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const u32x2 a = swap32(v);
    return bits_f32(a[0]) + bits_f32(a[1]);
}
__device__ __forceinline__ float base_of(float m) { return m == kNone ? 0.f : m; }

// Which of 64 keys are there and seen, a bit each.  A lane's byte of the mask is loaded a step before it is looked at: a wait for it would be
// one for what was requested in between too.
struct Seen {
    const RaggedArgs& a;
    const uint8_t* mask;  // of the lane's key among the first 64
    int left;             // keys from the lane's on
    uint8_t byte = 1;
    __device__ __forceinline__ Seen(const RaggedArgs& a, const RaggedItem& it, int first, int lane) : a(a) { start(it, first, lane); }
    __device__ __forceinline__ void start(const RaggedItem& it, int first, int lane) {
        mask = a.key_mask + it.k_row + first + lane;
        left = it.k_end - first - lane;
        if (a.key_mask && left > 0) byte = load_global<uint8_t>(mask);
    }
    // the bits of 64 keys; those looked at next time begin `step` keys on
    __device__ __forceinline__ uint64_t next(int step) {
        const uint64_t bits = __ballot(left > 0 && byte != 0);
        left -= step;
        mask += step;
        if (a.key_mask && left > 0) byte = load_global<uint8_t>(mask);
        return bits;
    }
};
// and by a query row at place `pos`
__device__ __forceinline__ uint64_t seen_from(uint64_t seen, int first, int pos, int causal) {
    if (!causal) return seen;
    const int last = pos - first;  // the last one that it sees
    return last >= 63 ? seen : last < 0 ? 0 : seen & ((2ull << last) - 1);
}

// ---- bias: in LDS by key - query + max_distance + kMargin.  Beyond both ends there are kMargin places more, so that a tile of 32 x 32 that
// touches the range needs no limits; one that does not has a single bucket ----
constexpr int kMargin = kAttnMargin;
__device__ __forceinline__ int bias_places(const RaggedArgs& a) { return a.span + 2 * kMargin; }
template <typename T> __device__ __forceinline__ void bias_to_lds(const RaggedArgs& a, float* w, int head) {
    for (int i = threadIdx.x; i < bias_places(a); i += blockDim.x) {
        const int bucket = a.bucket_of[min(max(i - kMargin, 0), a.span - 1)];
        const float b = to_f32(load_global<T>(static_cast<const T*>(a.bias) + (int64_t)bucket * a.heads + head));
        // a finite entry stays one, times log2 e too: minus infinity is for keys that are not seen
        w[i] = fabsf(b) < -kNone ? fminf(fmaxf(kLog2e * b, -__FLT_MAX__), __FLT_MAX__) : b;
    }
}
// Rows all of whose keys have a large bias, one that is as good as a mask where there are others.  What a float32 of that size is off by is no small
// part of a weight exp(s - lse): from -1e7 on the weights of such a row are off by whole factors.  The forward kernel is not concerned: its sum is one of its own
// weights.  The gradients' take maximum and log of the sum apart for rows whose lse is beyond a thousand; up to there it is off by 2^-14.
__device__ __forceinline__ bool is_large(float lse) { return fabsf(lse) > 1024.f && fabsf(lse) < -kNone; }
// The place of the first of 32 keys from `key` on and the first of 32 queries from `pos` on
enum { kTouches, kAllFar, kAllNear };
__device__ __forceinline__ int bias_region(const RaggedArgs& a, int key, int pos, int& at) {
    at = key - pos + a.max_distance;
    const int region = at + 31 <= 0 ? kAllFar : at - 31 >= a.span - 1 ? kAllNear : kTouches;
    at += kMargin;
    return region;
}
// s += bias; STEP 1: the lane is a query (its number r), elements are keys; -1: the other way about
template <int STEP> __device__ __forceinline__ void add_bias(f32x16& s, const RaggedArgs& a, const float* w, int key, int pos, int r, int h) {
    int at;
    const int region = bias_region(a, key, pos, at);
    if (region != kTouches) {
        const float b = w[region == kAllFar ? 0 : bias_places(a) - 1];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += b;
        return;
    }
    at += STEP * (4 * h - r);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] += w[at + STEP * (8 * (i >> 2) + (i & 3))];
}
// Sums of a tile's elements (lane = query) by distance, key - query = 4 h - y - 16 + 16 t for lane y of a 16-lane row: the elements of
// key 8 g + e are shifted along the row by that many lanes (an operand's modifier, not an instruction) so that one distance, modulo 16,
// stays in a lane; what leaves the row at one end and comes in at the other is 16 further.  (Adding every element to LDS, which
// takes its lanes' atomics one by one: dQ's kernel 241 us instead of 143, with the plain third product, on the
// long batch of its own.)
template <int K> __device__ __forceinline__ void add_shifted(float v, float* sum) {
    constexpr int n = K & 15, m = K >> 4;
    if constexpr (n == 0) {
        sum[m] += v;
    } else {
        sum[m] += dpp_mov<0x100 + n>(v);           // from lane y + n
        sum[m + 1] += dpp_mov<0x110 + 16 - n>(v);  // from lane y + n - 16
    }
}
// Adds the gradients of a tile (lane = query) to sums by distance.  mine: this lane half's own sums, so that no two lanes of an
// instruction meet and every sum has one order; far, near: of tiles beyond the ends, kept by lane.
__device__ __forceinline__ void add_distances(const f32x16& ds, const RaggedArgs& a, float* mine, float& far, float& near, int key, int pos, int lane) {
    int at;
    const int region = bias_region(a, key, pos, at);
    if (region != kTouches) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += ds[i];
        if (region == kAllFar) far += sum;
        else near += sum;
        return;
    }
    float sum[3] = {0.f, 0.f, 0.f};
    add_shifted<0>(ds[0], sum), add_shifted<1>(ds[1], sum), add_shifted<2>(ds[2], sum), add_shifted<3>(ds[3], sum);
    add_shifted<8>(ds[4], sum), add_shifted<9>(ds[5], sum), add_shifted<10>(ds[6], sum), add_shifted<11>(ds[7], sum);
    add_shifted<16>(ds[8], sum), add_shifted<17>(ds[9], sum), add_shifted<18>(ds[10], sum), add_shifted<19>(ds[11], sum);
    add_shifted<24>(ds[12], sum), add_shifted<25>(ds[13], sum), add_shifted<26>(ds[14], sum), add_shifted<27>(ds[15], sum);
    // the second row's queries are 16 on: its sums belong to the first's of one less
    const u32x2 s0 = swap16(sum[0]), s1 = swap16(sum[1]), s2 = swap16(sum[2]);
    const bool second = lane & 16;
    const float one = second ? bits_f32(s1[0]) + bits_f32(s2[1]) : bits_f32(s0[1]);
    const float two = second ? bits_f32(s2[0]) : bits_f32(s0[0]) + bits_f32(s1[1]);
    float* const to = mine + at + 4 * (lane >> 5) - (lane & 15) - 16 + (second ? 32 : 0);
    __hip_atomic_fetch_add(to, one, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __hip_atomic_fetch_add(to + 16, two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// nothing is moved across by the compiler
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// ends a phase of eight 32 x 32 products among which the vector instructions are dealt out
template <int FIRST, int READS, int EACH> __device__ __forceinline__ void woven() {
    if constexpr (FIRST > 0) __builtin_amdgcn_sched_group_barrier(0x2, FIRST, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // a product
        if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);  // reads of LDS
        if constexpr (EACH > 0) __builtin_amdgcn_sched_group_barrier(0x2, EACH, 0);  // vector instructions
    }
    phase();
}

// Keeps what a branch computes from `v` in the branch: the compiler would rather do it always than jump
__device__ __forceinline__ void rarely(uint32_t& v) { asm volatile("" : "+v"(v)); }

// scores of a tile (lane = query) from its products: without a bias they stay unscaled (times scale2 later), with one they are whole;
// those of keys that are not seen (bits of `seen`) out of the way
template <bool BIAS>
__device__ __forceinline__ void finish_scores(f32x16& s, const RaggedArgs& a, float scale2, const float* w, uint32_t seen, int key, int pos, int r, int h) {
    if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= scale2;
        add_bias<1>(s, a, w, key, pos, r, h);
    }
    if (__ballot(seen != 0xffffffffu) != 0) {
        uint32_t mine = seen >> (4 * h);
        rarely(mine);
#pragma unroll
        for (int i = 0; i < 16; ++i) {  // (a bit spread over 32, and a choice by bits: no condition codes)
            const unsigned yes = (unsigned)__builtin_amdgcn_sbfe((int)mine, 8 * (i >> 2) + (i & 3), 1);
            const float x = s[i];
            s[i] = bits_f32((__builtin_bit_cast(unsigned, x) & yes) | (__builtin_bit_cast(unsigned, kNone) & ~yes));
        }
    }
}
// exp of a score less `base`, both times log2 e
template <bool BIAS> __device__ __forceinline__ float weight_of(float s, float scale2, float base) {
    return __builtin_amdgcn_exp2f(BIAS ? s - base : fmaf(s, scale2, -base));
}

// Softmax of a lane's row in passing: maximum so far (times log2 e), and the lane half's share of the sum
struct Running {
    float m = kNone, l = 0.f;
    template <int TILES> __device__ __forceinline__ float scale_to(float m_tile, f32x16* acc) {
        const float m_new = fmaxf(m, m_tile), base = base_of(m_new), alpha = __builtin_amdgcn_exp2f(m - base);
        l *= alpha;
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t] *= alpha;
        m = m_new;
        return base;
    }
};
// one tile of scores to weights; the sum goes to l
template <bool BIAS> __device__ __forceinline__ void to_weights(f32x16& s, float scale2, float base, float& l) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = weight_of<BIAS>(s[i], scale2, base);
    l += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])) + (((s[8] + s[9]) + (s[10] + s[11])) + ((s[12] + s[13]) + (s[14] + s[15])));
}
__device__ __forceinline__ float max_of(const f32x16& s) {
    float m = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
    return m;
}

template <int TILES> __device__ __forceinline__ void clear(f32x16* acc) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
}

// Where a wavefront's part of the walk over the keys ends: it has no rows, or they see no further
__device__ __forceinline__ int end_of(const RaggedArgs& a, const RaggedItem& it, int count, int pos) {
    return count == 0 ? it.k_begin : a.causal ? min(it.k_end, max(it.k_begin, pos + count)) : it.k_end;
}

// A workgroup's walk over the keys, kStep of them a step: keys and values from memory to LDS (rows of keys, then of values), two
// steps' worth: one is worked on while the other is on its way.
template <typename T, int D> struct Steps {
    typedef Rows<T, D> R;
    static constexpr int kBuf = 2 * R::kStep * R::kPitch;
    const RaggedArgs& a;
    const RaggedItem& it;
    const char *kp, *vp;
    char* lds;
    int lane;
    RowFeed<T, D, R::kStep> feed;
    Seen bits;
    uint64_t seen = 0, seen_next = 0;  // of the step at hand and of the one on its way
    int buf = 1;
    bool there = false;  // all of the walk is in LDS
    __device__ __forceinline__ Steps(const RaggedArgs& a, const RaggedItem& it, int kv_head, char* lds, int wave, int lane)
        : a(a), it(it), kp(a.k.p + it.k_row * a.k.row + kv_head * a.k.head), vp(a.v.p + it.k_row * a.v.row + kv_head * a.v.head), lds(lds), lane(lane),
          feed(lds, wave, lane), bits(a, it, it.k_begin, lane) {}
    // requests the step of keys k0 on, into the buffer that is not at hand
    __device__ __forceinline__ void fetch(int k0) {
        if (k0 >= it.k_end) return;
        const int count = it.k_end - k0, to = (buf ^ 1) * kBuf;
        seen_next = a.key_mask ? bits.next(R::kStep) : count >= 64 ? ~0ull : (1ull << count) - 1;
        if (there) return;
        const char *ks = kp + k0 * a.k.row, *vs = vp + k0 * a.v.row;
        if (a.key_mask && (seen_next & R::kAll) != R::kAll) {
            feed.load_seen(ks, (int)a.k.row, seen_next, a.zeros, to);
            feed.load_seen(vs, (int)a.v.row, seen_next, a.zeros, to + kBuf / 2);
        } else {
            feed.load(ks, (int)a.k.row, count, to);
            feed.load(vs, (int)a.v.row, count, to + kBuf / 2);
        }
    }
    // from the beginning again; everyone is done with the last step, and none is on its way.  whole: both buffers still hold a walk of two steps
    __device__ __forceinline__ void again(bool whole) {
        bits.start(it, it.k_begin, lane);
        buf = 1;
        there = whole;
        fetch(it.k_begin);
    }
    // everyone is done with the step at hand; the one on its way is at hand
    __device__ __forceinline__ void next() {
        loads_done_barrier();
        buf ^= 1;
        seen = seen_next;
    }
    __device__ __forceinline__ const char* keys() const { return lds + buf * kBuf; }
    __device__ __forceinline__ const char* values() const { return lds + buf * kBuf + kBuf / 2; }
};

}  // namespace

// ---------------------------------------------------------------- forward, many rows
// A workgroup takes 128 query rows of a head, 32 a wavefront, and walks the keys.  PAIR: it takes 64 rows, and two wavefronts share 32 of them,
// each with 32 keys of a step.  Scores are computed transposed (a lane is a query), so that a lane holds half a row's weights
// and they enter the second product from where they are.  128 utterances of 448 rows and 512 keys take 199 to 212 us; of the 202 that an earlier form
// took, 100 were the two products (their rate is a large product's), 30 the softmax in between, 35 the wait for keys and values and 39 starts and ends.  Two
// workgroups share a compute unit to cover one's waits with the other's products, which is why a wavefront has 256 registers and 32 rows: with 64 rows
// and all registers it was 258 us against the same form's 184.  Short batches are bound by starts and ends, a single round of workgroups.
template <typename T, int D, bool BIAS, bool PAIR> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_forward_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kJoin = 2 * 64 * R::kTiles * 64 + 1024;  // two wavefronts' sums, and their maxima
    constexpr int kSub = PAIR ? 1 : R::kStep / 32;  // 32-key tiles of a step
    static_assert(!PAIR || R::kStep == 64, "a tile for each of two");
    float* const w = reinterpret_cast<float*>(lds + 2 * Steps<T, D>::kBuf);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const RaggedItem it = a.items[blockIdx.x / a.heads];
    const int group = PAIR ? wave & 1 : wave, tile = PAIR ? wave >> 1 : 0;  // which rows, which keys of a step
    const int head = blockIdx.x % a.heads, row0 = it.q_row + 32 * group, count = min(max(it.rows - 32 * group, 0), 32), pos = it.pos + 32 * group;
    Steps<T, D> step(a, it, head / a.share, lds, wave, lane);
    step.fetch(it.k_begin);
    RowFrag<T, D> q;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, r < count, h);
    if constexpr (BIAS) bias_to_lds<T>(a, w, head);
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    Running run;
    const float scale2 = a.scale * kLog2e;
    const int mine_end = end_of(a, it, count, pos);
    int k0 = it.k_begin;
    for (; k0 < mine_end; k0 += R::kStep) {
        step.next();
        step.fetch(k0 + R::kStep);
        f32x16 s[kSub];
        AsRows<T, D> k[kSub];
        AsColumns<T, D> v[kSub];
#pragma unroll
        for (int u = 0; u < kSub; ++u) k[u].load(step.keys(), 32 * (tile + u), lane);
        phase();
        k[0].dot(s[0], q);
        phase();
        v[0].load(step.values(), 32 * tile, lane);
        phase();
        if constexpr (kSub > 1) k[1].dot(s[1], q);
        const uint64_t seen = seen_from(step.seen, k0, pos + r, a.causal);
        float top = kNone;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            finish_scores<BIAS>(s[u], a, scale2, w, (uint32_t)(seen >> (32 * (tile + u))), k0 + 32 * (tile + u), pos, r, h);
            top = fmaxf(top, max_of(s[u]));
        }
        top = max_halves(top);
        const float base = run.scale_to<R::kTiles>(BIAS ? top : top * scale2, acc);
        to_weights<BIAS>(s[0], scale2, base, run.l);
        phase();
        if constexpr (kSub > 1) v[1].load(step.values(), 32, lane);
        phase();
        v[0].add(acc, s[0]);
        if constexpr (kSub > 1) {
            to_weights<BIAS>(s[1], scale2, base, run.l);
            v[1].add(acc, s[1]);
        }
    }
    for (; k0 < it.k_end; k0 += R::kStep) {  // the other wavefronts' steps
        step.next();
        step.fetch(k0 + R::kStep);
    }
    float l = sum_halves(run.l);
    if constexpr (PAIR) {  // the second wavefront's maximum and sums join the first's
        lds_barrier();
        float* const given = reinterpret_cast<float*>(lds) + (group * 64 + lane) * 4;
        float2* const ml = reinterpret_cast<float2*>(lds + kJoin - 1024) + group * 64 + lane;
        if (tile == 1) {
            *ml = float2{run.m, l};
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4*>(given + (t * 4 + g) * 512) = f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
        }
        lds_barrier();
        if (tile == 1) return;
        const float m = fmaxf(run.m, ml->x), alpha = __builtin_amdgcn_exp2f(run.m - base_of(m)), beta = __builtin_amdgcn_exp2f(ml->x - base_of(m));
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(given + (t * 4 + g) * 512);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][4 * g + e] = acc[t][4 * g + e] * alpha + v[e] * beta;
            }
        l = l * alpha + ml->y * beta;
        run.m = m;
    }
    if (it.part < 0) {
        if constexpr (!PAIR) lds_barrier();
        store_tile<T, D>(acc, l > 0.f ? 1.f / l : l, lds + (PAIR ? kJoin : 0) + group * 32 * R::kPitch, a.o.p + (int64_t)row0 * a.o.row + head * a.o.head, a.o.row, count, lane);
        if (h == 0 && r < count) a.lse[(int64_t)(row0 + r) * a.heads + head] = kLn2 * (run.m + __builtin_amdgcn_logf(l));
    } else if (r < count) {
        const int64_t at = ((int64_t)it.part * a.heads + head) * (PAIR ? kAttnPair : kAttnRows) + 32 * group + r;
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                store4(a.part_o + at * D + 32 * t + 8 * g + 4 * h, f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]});
        if (h == 0) a.part_ml[at] = float2{run.m, l};
    }
}

// ---------------------------------------------------------------- forward, few rows
// A workgroup takes up to 32 query rows of a head; its four wavefronts take 32 keys each in turn, through rows of LDS of their own, and
// join their sums at the end.  The matrix cores are mostly idle here: what counts is that keys and values stream.  Bound by memory: one row for
// each of 256 utterances, 31 792 keys of 8 heads of 128, 131 MB in 26.8 us, 4.9 TB/s (a large copy: 5.1); 64 sequences with 13 696 keys
// in a cache of 448, with bias, 56 MB in 14.5 us.  One utterance of 100 frames takes 5.3 us, which is a launch and three trips to memory.
template <typename T, int D, bool BIAS> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_few_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kMine = 2 * 32 * R::kPitch;
    float* const w = reinterpret_cast<float*>(lds + 4 * kMine);
    __shared__ float2 ml[4][32];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const RaggedItem it = a.items[blockIdx.x / a.heads];
    const int head = blockIdx.x % a.heads, row0 = it.q_row, count = it.rows, pos = it.pos;
    const int64_t k_head = (int64_t)(head / a.share) * a.k.head, v_head = (int64_t)(head / a.share) * a.v.head;
    const char* const kp = a.k.p + it.k_row * a.k.row + k_head;
    const char* const vp = a.v.p + it.k_row * a.v.row + v_head;
    char* const kb = lds + wave * kMine;
    char* const vb = kb + kMine / 2;
    RowStage<T, D, 32> ks, vs;
    uint64_t seen = 0;
    Seen bits(a, it, it.k_begin + 32 * wave, lane);
    auto fetch = [&](int k0) {
        seen = bits.next(128);
        ks.load(kp + k0 * a.k.row, (int)a.k.row, it.k_end - k0, seen, lane);
        vs.load(vp + k0 * a.v.row, (int)a.v.row, it.k_end - k0, seen, lane);
    };
    int k0 = it.k_begin + 32 * wave;
    if (k0 < it.k_end) fetch(k0);
    RowFrag<T, D> q;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, r < count, h);
    if constexpr (BIAS) {
        bias_to_lds<T>(a, w, head);
        lds_barrier();
    }
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    Running run;
    const float scale2 = a.scale * kLog2e;
    for (; k0 < it.k_end; k0 += 128) {
        ks.store(kb, lane);
        vs.store(vb, lane);
        other_lanes_wrote();
        const uint32_t mine = (uint32_t)seen_from(seen, k0, pos + r, a.causal);
        if (k0 + 128 < it.k_end) fetch(k0 + 128);
        f32x16 s;
        AsRows<T, D> k;
        k.load(kb, 0, lane);
        k.dot(s, q);
        finish_scores<BIAS>(s, a, scale2, w, mine, k0, pos, r, h);
        const float top = max_halves(max_of(s)), base = run.template scale_to<R::kTiles>(BIAS ? top : top * scale2, acc);
        to_weights<BIAS>(s, scale2, base, run.l);
        AsColumns<T, D> v;
        v.load(vb, 0, lane);
        v.add(acc, s);
        other_lanes_wrote();
    }
    // join: maximum, then the sums scaled to it
    float l = sum_halves(run.l);
    if (h == 0) ml[wave][r] = float2{run.m, l};
    __syncthreads();
    float m = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, ml[i][r].x);
    const float alpha = __builtin_amdgcn_exp2f(run.m - base_of(m));
    float* const sums = reinterpret_cast<float*>(lds);  // [4][count][D]; the wavefronts' rows are done with
    if (r < count) {
#pragma unroll
        for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(sums + (wave * count + r) * D + 32 * t + 8 * g + 4 * h) =
                    f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]} * alpha;
    }
    __syncthreads();
    for (int i = tid; i < count * (D / 4); i += 256) {
        const int row = i / (D / 4), c = i % (D / 4) * 4;
        float top = kNone, total = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, ml[j][row].x);
#pragma unroll
        for (int j = 0; j < 4; ++j) total += ml[j][row].y * __builtin_amdgcn_exp2f(ml[j][row].x - base_of(top));
        f32x4 v = *reinterpret_cast<const f32x4*>(sums + row * D + c);
#pragma unroll
        for (int j = 1; j < 4; ++j) v += *reinterpret_cast<const f32x4*>(sums + (j * count + row) * D + c);
        if (it.part < 0) {
            v *= total > 0.f ? 1.f / total : total;
            put4(a.o.p + (int64_t)(row0 + row) * a.o.row + head * a.o.head + c * sizeof(T), v, (const T*)nullptr);
            if (c == 0) a.lse[(int64_t)(row0 + row) * a.heads + head] = kLn2 * (top + __builtin_amdgcn_logf(total));
        } else {
            const int64_t at = ((int64_t)it.part * a.heads + head) * kAttnFew + row;
            store4(a.part_o + at * D + c, v);
            if (c == 0) a.part_ml[at] = float2{top, total};
        }
    }
}

// ---------------------------------------------------------------- parts of rows whose keys were split
// Bound by memory, the parts' sums mostly from the caches that they were just written to: 5 utterances of 1 757 rows and 2000 to 6000 keys 9.5 us
// behind 64 us of the walks.  Parts stay float32: a sum of parts is rounded once, as an unsplit row's is.
template <typename T, int D> __global__ __launch_bounds__(256) void attn_join_kernel(RaggedArgs a, int tile_rows) {
    const RaggedJoin j = a.joins[blockIdx.x];
    const int head = blockIdx.y, per = D / 4, at = blockIdx.z * 256 + threadIdx.x;
    if (at >= j.rows * per) return;
    const int row = at / per, c = at % per * 4;
    const int64_t first = ((int64_t)j.part * a.heads + head) * tile_rows + row, step = (int64_t)a.heads * tile_rows;
    float m = kNone;
    for (int i = 0; i < j.n_parts; ++i) m = fmaxf(m, a.part_ml[first + i * step].x);
    float l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < j.n_parts; ++i) {
        const float2 p = a.part_ml[first + i * step];
        const float alpha = __builtin_amdgcn_exp2f(p.x - base_of(m));
        l += p.y * alpha;
        v += load4(a.part_o + (first + i * step) * D + c) * alpha;
    }
    v *= l > 0.f ? 1.f / l : l;
    put4(a.o.p + (int64_t)(j.q_row + row) * a.o.row + head * a.o.head + c * sizeof(T), v, (const T*)nullptr);
    if (c == 0) a.lse[(int64_t)(j.q_row + row) * a.heads + head] = kLn2 * (m + __builtin_amdgcn_logf(l));
}

// ---------------------------------------------------------------- query gradients, delta, and the bias's
// The forward kernel's walk with two products to a tile of scores (K Q^T and V dO^T, transposed, a lane being a query) and one
// more for dQ, which in bfloat16 is made with what rounding took off dS as well (280 us on the long batch; an earlier form 286, 250 without it).
// delta: from the output as it was stored, whose rounding to bfloat16 goes into every dS of the row, or as the sum of P dP over the keys, in a walk of
// its own before: five products instead of three.  The rounding counts where few keys have the weight, as the output is as large as a value then, and in
// the bias's gradient, where it adds up over a bucket: self-attention of 8 to 34 positions has dQ off by 0.0025 to 0.0031 and dw by up to 0.0032 with it, and by
// the 0.0017 of the result's own rounding without.  So bfloat16 makes the first walk if there is a bias (long batch of its own 168 to 176 us, 154 without) and
// where the keys, up to 128, stay in LDS for the second (short batch 28.5 us, 28.7 without).  Other walks take the stored output, with
// 300 keys and more dQ is 0.0017 to 0.0018 off (long batch 280 us, 390 with two walks; short 28.5, with two walks for all 36.9).  By float64 arithmetic with
// an output so rounded it would be 0.003 to 0.005 off if attention were so sharp that a row has the weight of two or three keys among 448.
// For the key gradients' kernel delta is left without that error in any case: a row's dS add up to 0, so what they do add up to is what delta lacks.
// Bound like the forward kernel.  Fragments are read where they are used: read one product ahead, as in the kernel below, they need more than 256
// registers (424 to 796 us on the long batch, with the plain third product).
namespace {

// Maximum (times log2 e) and sum of a lane's row, as the forward kernel finds them, in a walk of its own; the first step is on its way, before and after.
// Rows that are not there have weights that nobody looks at.
template <typename T, int D, bool PAIR>
__device__ __forceinline__ float2 top_and_sum(const RaggedArgs& a, const RaggedItem& it, Steps<T, D>& step, const RowFrag<T, D>& q, const float* w, float2* joined,
                                              int mine_end, int pos, int tile, int wave, int lane) {
    typedef Rows<T, D> R;
    const int r = lane & 31, h = lane >> 5;
    const float scale2 = a.scale * kLog2e;
    float m = kNone, l = 0.f;
    for (int k0 = it.k_begin; k0 < it.k_end; k0 += R::kStep) {
        step.next();
        step.fetch(k0 + R::kStep);
        if (k0 >= mine_end) continue;
        const uint64_t seen = seen_from(step.seen, k0, pos + r, a.causal);
#pragma unroll 1
        for (int u = 0; u < (PAIR ? 1 : R::kStep / 32); ++u) {
            const int key = 32 * (tile + u);
            f32x16 s;
            AsRows<T, D> k;
            k.load(step.keys(), key, lane);
            k.dot(s, q);
            finish_scores<true>(s, a, scale2, w, (uint32_t)(seen >> key), k0 + key, pos, r, h);
            const float top = fmaxf(m, max_of(s)), base = base_of(top);
            l *= __builtin_amdgcn_exp2f(m - base);
            m = top;
            to_weights<true>(s, scale2, base, l);
        }
    }
    auto join = [&](float m2, float l2) {
        const float top = fmaxf(m, m2), base = base_of(top);
        l = l * __builtin_amdgcn_exp2f(m - base) + l2 * __builtin_amdgcn_exp2f(m2 - base);
        m = top;
    };
    const u32x2 ms = swap32(m), ls = swap32(l);
    m = bits_f32(ms[0]), l = bits_f32(ls[0]);
    join(bits_f32(ms[1]), bits_f32(ls[1]));
    lds_barrier();
    if constexpr (PAIR) {  // the two wavefronts with the same rows
        joined[wave * 64 + lane] = float2{m, l};
        lds_barrier();
        const float2 first = joined[(wave & 1) * 64 + lane], second = joined[(wave | 2) * 64 + lane];
        m = first.x, l = first.y;  // both join them in the same order
        join(second.x, second.y);
        lds_barrier();
    }
    step.again(false);
    return float2{m, l};
}

}  // namespace

template <typename T, int D, bool BIAS, bool PAIR> __global__ __launch_bounds__(256, (2 - Rows<T, D>::kWide)) void attn_dq_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    extern __shared__ __align__(16) char lds[];
    constexpr int kJoin = 2 * 64 * R::kTiles * 64 + 512;  // two wavefronts' sums, and of their rows' delta
    static_assert(!PAIR || R::kStep == 64, "a tile for each of two");
    float* const w = reinterpret_cast<float*>(lds + 2 * Steps<T, D>::kBuf);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    const int places = bias_places(a);
    float* const sums = w + places;  // [wavefront, half][places]
    const int item = blockIdx.x / a.heads;
    const RaggedItem it = a.items[item];
    const int group = PAIR ? wave & 1 : wave, tile = PAIR ? wave >> 1 : 0;  // which rows, which keys of a step
    const int head = blockIdx.x % a.heads, row0 = it.q_row + 32 * group, count = min(max(it.rows - 32 * group, 0), 32), pos = it.pos + 32 * group;
    Steps<T, D> step(a, it, head / a.share, lds, wave, lane);
    step.fetch(it.k_begin);
    const bool live = r < count;
    RowFrag<T, D> q, d_o;
    q.load(a.q.p + (int64_t)(row0 + r) * a.q.row + head * a.q.head, live, h);
    d_o.load(a.d_o.p + (int64_t)(row0 + r) * a.d_o.row + head * a.d_o.head, live, h);
    constexpr bool kRounded = sizeof(T) == 2;  // outputs are
    const bool resident = it.k_end - it.k_begin <= 2 * R::kStep, twice = kRounded && (BIAS || resident);  // (the rule's figures are above)
    float delta = 0.f, rest = 0.f;
    if (!twice) {
        RowFrag<T, D> o;
        o.load(a.o.p + (int64_t)(row0 + r) * a.o.row + head * a.o.head, live, h);
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 16 / (int)sizeof(T); ++e) delta += to_f32((T)o.c[s][e]) * to_f32((T)d_o.c[s][e]);
        delta = sum_halves(delta);
    }
    // a row that sees nothing has lse -inf, and none of its keys' bits are set: its weights become 0 by way of the scores; those of a row that is
    // not there are 2^-inf, as its scores are the bias, of any size
    const float lse = live ? a.lse[(int64_t)(row0 + r) * a.heads + head] : 0.f, scale2 = a.scale * kLog2e;
    float base = live ? base_of(kLog2e * lse) : -kNone;
    const int mine_end = end_of(a, it, count, pos);
    bool large = false;  // the workgroup has rows with a large lse: scores are taken from `tops`, and `base` is what is left to take away
    __shared__ float tops[BIAS ? 4 * 32 : 1], exchanged[BIAS || (PAIR && kRounded) ? 4 * 32 : 1];  // (together what launch() leaves of a compute unit's LDS)
    if constexpr (BIAS) {
        bias_to_lds<T>(a, w, head);
        for (int i = tid; i < 8 * places; i += 256) sums[i] = 0.f;
        const bool mine = __ballot(is_large(lse)) != 0;
        if (lane == 0) exchanged[wave] = mine ? 1.f : 0.f;
        lds_barrier();
        large = __ballot(exchanged[lane & 3] != 0.f) != 0;
        if (large) {
            float2 of = top_and_sum<T, D, PAIR>(a, it, step, q, w, reinterpret_cast<float2*>(lds), mine_end, pos, tile, wave, lane);
            of = is_large(lse) ? float2{of.x, of.y > 0.f ? __builtin_amdgcn_logf(of.y) : 0.f} : float2{base, 0.f};
            if (h == 0) tops[wave * 32 + r] = of.x;
            other_lanes_wrote();
            base = of.y;
            if (is_large(lse) && h == 0 && tile == 0) a.large[(int64_t)(row0 + r) * a.heads + head] = of;
        }
    }
    // the step at hand: which keys the lane's row sees (rows that are not there have weights of zero without a mask), and of a tile the weights' scores and dP
    auto seen_at = [&](int k0) { return live ? seen_from(step.seen, k0, pos + r, a.causal) : ~0ull; };
    auto products = [&](f32x16& s, f32x16& dp, int k0, int key, uint64_t seen) {
        AsRows<T, D> k, v;
        k.load(step.keys(), key, lane);
        k.dot(s, q);
        v.load(step.values(), key, lane);
        v.dot(dp, d_o);
        finish_scores<BIAS>(s, a, scale2, w, (uint32_t)(seen >> key), k0 + key, pos, r, h);
        if (BIAS && large) {
            const float top = tops[wave * 32 + r];
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = fminf(s[i] - top, 0.f);
        }
    };
    if constexpr (kRounded) {
        if (twice) {  // delta, from a walk of its own
            for (int k0 = it.k_begin; k0 < it.k_end; k0 += R::kStep) {
                step.next();
                step.fetch(k0 + R::kStep);
                if (k0 >= mine_end) continue;
                const uint64_t seen = seen_at(k0);
#pragma unroll 1
                for (int u = 0; u < (PAIR ? 1 : R::kStep / 32); ++u) {
                    f32x16 s, dp;
                    products(s, dp, k0, 32 * (tile + u), seen);
#pragma unroll
                    for (int i = 0; i < 16; ++i) delta = fmaf(weight_of<BIAS>(s[i], scale2, base), dp[i], delta);
                }
            }
            delta = sum_halves(delta);
            lds_barrier();
            if constexpr (PAIR) {  // two wavefronts have the same rows
                if (h == 0) exchanged[wave * 32 + r] = delta;
                lds_barrier();
                delta = exchanged[group * 32 + r] + exchanged[(group + 2) * 32 + r];
            }
            step.again(resident);
        }
    }
    f32x16 acc[R::kTiles];
    clear<R::kTiles>(acc);
    float far = 0.f, near = 0.f;
    int k0 = it.k_begin;
    for (; k0 < mine_end; k0 += R::kStep) {
        step.next();
        step.fetch(k0 + R::kStep);
        const uint64_t seen = seen_at(k0);
#pragma unroll
        for (int u = 0; u < (PAIR ? 1 : R::kStep / 32); ++u) {
            const int key = 32 * (tile + u);
            f32x16 s, dp;
            AsColumns<T, D> kt;
            products(s, dp, k0, key, seen);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = weight_of<BIAS>(s[i], scale2, base) * (dp[i] - delta);
                if constexpr (!(kRounded && BIAS)) rest += s[i];
            }
            if constexpr (BIAS) add_distances(s, a, sums + (2 * wave + h) * places, far, near, k0 + key, pos, lane);
            phase();
            kt.load(step.keys(), key, lane);
            kt.add_finely(acc, s);
            phase();
        }
    }
    for (; k0 < it.k_end; k0 += R::kStep) {  // the other wavefronts' steps
        step.next();
        step.fetch(k0 + R::kStep);
    }
    lds_barrier();
    rest = sum_halves(rest);
    if constexpr (PAIR) {  // the second wavefront's sums join the first's
        float* const given = reinterpret_cast<float*>(lds) + (group * 64 + lane) * 4;
        float* const rests = reinterpret_cast<float*>(lds + kJoin - 512) + group * 64 + lane;
        if (tile == 1) {
            *rests = rest;
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4*>(given + (t * 4 + g) * 512) = f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
        }
        lds_barrier();
        if (tile == 0) {
            rest += *rests;
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(given + (t * 4 + g) * 512);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][4 * g + e] += v[e];
                }
        }
    }
    if (tile == 0) {
        if (live && h == 0) a.delta[(int64_t)(row0 + r) * a.heads + head] = delta + rest;
        store_tile<T, D>(acc, a.scale, lds + (PAIR ? kJoin : 0) + group * 32 * R::kPitch, a.dq.p + (int64_t)row0 * a.dq.row + head * a.dq.head, a.dq.row, count, lane);
    }
    if constexpr (BIAS) {
        // the ends' sums by wavefront, then the eight sums of a distance, then a bucket's distances, which lie side by side
        far = wave_sum(far);
        near = wave_sum(near);
        lds_barrier();
        if (lane == 0) {
            sums[2 * wave * places] += far;
            sums[2 * wave * places + places - 1] += near;
        }
        lds_barrier();
        for (int i = tid; i < places; i += 256) {
            float v = 0.f;
            for (int j = 0; j < 8; ++j) v += sums[j * places + i];
            w[i] = v;
        }
        lds_barrier();
        float* const out = a.part_bias + ((int64_t)item * a.heads + head) * a.buckets;
        for (int b = tid; b < a.buckets; b += 256) {
            float v = 0.f;
            const int2 range = a.bucket_range[b];
            for (int i = range.x; i < range.y; ++i) v += w[i];
            out[b] = v;
        }
    }
}

// ---------------------------------------------------------------- key and value gradients
namespace {

// Bias gradient: the items' sums of one bucket and head, by a wavefront
template <typename T> __device__ __forceinline__ void reduce_bias(const RaggedArgs& a, int which, int lane) {
    if (which >= a.buckets * a.heads) return;
    const int b = which / a.heads, head = which % a.heads;
    float v = 0.f;
    for (int i = lane; i < a.bias_items; i += 64) v += a.part_bias[((int64_t)i * a.heads + head) * a.buckets + b];
    v = wave_sum(v);
    if (lane == 0) static_cast<T*>(a.d_bias)[which] = from_f32<T>(v);
}

}  // namespace

constexpr int kLargeFlags = 4;  // places of LDS

// A workgroup takes 128 keys of a key head, 32 a wavefront (a lane being a key), and walks the query rows of all heads that share it.
// PAIR: it takes 64 keys, and two wavefronts share 32 of them, each with 32 rows of a step.  Four products to a tile and no sum over
// workgroups: what heads share is added up here, in order.
// Two accumulators of 32 keys and the keys and values themselves take 192 registers, so that a wavefront has a SIMD to itself and nothing else
// covers its waits: operands are requested one product ahead, and their reads and the vector instructions stand among the matrix
// instructions (384 us on the long batch; requested at their use 426).  128 utterances of 448 rows and 512 keys take 364 to 382 us; of an earlier form's 400, 331 remain without any
// request to memory in the loop, 74 of them starts and ends.  Slower: two workgroups a compute unit in 256 registers each 467, eight wavefronts
// with keys and values in LDS 432, 64 keys a wavefront 499; one workgroup a compute unit that goes on to the next task 401, and 38 instead of
// 28 us for short causal sequences, which do not end together then.
template <typename T, int D, bool SHAPED, bool PAIR> __global__ __launch_bounds__(256, 1) void attn_dkv_kernel(RaggedArgs a) {
    typedef Rows<T, D> R;
    constexpr int kRows = R::kStep, kBuf = 2 * kRows * R::kPitch, kTilesOf = PAIR ? 1 : kRows / 32;  // 32-row tiles of a step for a wavefront
    static_assert(!PAIR || kRows == 64, "a tile for each of two");
    extern __shared__ __align__(16) char lds[];
    float* const stats = reinterpret_cast<float*>(lds + 2 * kBuf);  // two buffers of [kRows] lse (times log2 e), [kRows] delta
    float* const tops = stats + 4 * kRows;                          // two of [kRows], of steps that have rows with a large lse:
    int* const large = reinterpret_cast<int*>(tops + 2 * kRows);    // whether these have; lse is what is left then to take away
    float* const w = tops + 2 * kRows + kLargeFlags;
    const int kv_heads = a.heads / a.share;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, h = lane >> 5;
    if ((int)blockIdx.x >= a.n_items * kv_heads) {  // behind the keys' workgroups: the bias's gradient
        if constexpr (SHAPED) reduce_bias<T>(a, (blockIdx.x - a.n_items * kv_heads) * 4 + wave, lane);
        return;
    }
    const RaggedItem it = a.items[blockIdx.x / kv_heads];
    const int kv_head = blockIdx.x % kv_heads, group = PAIR ? wave & 1 : wave, half = PAIR ? wave >> 1 : 0;  // which keys, which rows of a step
    const int count = min(max(it.rows - 32 * group, 0), 32), key0 = it.pos + 32 * group;
    const int64_t k_row0 = it.k_row + 32 * group;
    const RowFeed<T, D, kRows> feed(lds, wave, lane);
    int head = kv_head * a.share, buf = 1;
    float stat = 0.f;
    // requests the step of query rows q0 on, into the buffer that is not at hand
    auto fetch_stats = [&](int head, int q0) {
        const int n = it.k_end - q0;
        if (tid < 2 * kRows) {  // a row that is not there or sees nothing: its weights are 2^-inf
            const int row = tid & (kRows - 1);
            stat = tid < kRows ? -kNone : 0.f;
            if (row < n) {
                const int64_t at = (int64_t)(it.q_row + q0 + row) * a.heads + head;
                stat = tid < kRows ? a.lse[at] : a.delta[at];
            }
        }
    };
    auto put_stats = [&](int head, int q0) {
        if (tid >= 2 * kRows) return;
        const int to = buf ^ 1;
        float x = stat;
        if (tid < kRows) {
            x = kLog2e * stat;
            if (x == kNone) x = -kNone;
            if (SHAPED && a.span) {
                const bool some = __ballot(is_large(stat)) != 0;
                if (tid == 0) large[to] = some;
                if (some) {
                    float2 of = {x, 0.f};
                    if (is_large(stat)) of = a.large[(int64_t)(it.q_row + q0 + tid) * a.heads + head];
                    tops[to * kRows + tid] = of.x;
                    x = of.y;
                }
            }
        }
        stats[to * 2 * kRows + tid] = x;
    };
    if (it.k_begin < it.k_end) {
        feed.load(a.q.p + (int64_t)(it.q_row + it.k_begin) * a.q.row + head * a.q.head, (int)a.q.row, it.k_end - it.k_begin, 0);
        feed.load(a.d_o.p + (int64_t)(it.q_row + it.k_begin) * a.d_o.row + head * a.d_o.head, (int)a.d_o.row, it.k_end - it.k_begin, kBuf / 2);
        fetch_stats(head, it.k_begin);
    }
    bool live = r < count;
    if (a.key_mask && live) live = load_global<uint8_t>(a.key_mask + k_row0 + r) != 0;
    RowFrag<T, D> k, v;
    k.load(a.k.p + (k_row0 + r) * a.k.row + kv_head * a.k.head, live, h);
    v.load(a.v.p + (k_row0 + r) * a.v.row + kv_head * a.v.head, live, h);
    f32x16 dk[R::kTiles], dv[R::kTiles];
    clear<R::kTiles>(dk);
    clear<R::kTiles>(dv);
    const float scale2 = a.scale * kLog2e;
    // Small batches (pairs) with few rows: the roundings of a handful of weights do not average out (dK and dV off by up to 0.0026, where the result's own
    // rounding is 0.0017 and larger batches have 0.0023 to 0.0024), so their rest is multiplied too: 0.0017.  One utterance of 4 rows, both kernels of the backward
    // pass: 20.6 us, 19.5 without; 8 of 60 rows and 120 keys 18.7 and 18.4.  In all kernels: training steps of 64 short sequences with a bias 75.2 us, 72.9 so.
    constexpr bool kFine = sizeof(T) == 2 && PAIR;
    const bool fine = it.k_end - it.k_begin <= kRows;
    for (; head < (kv_head + 1) * a.share; ++head) {
        if (SHAPED && a.span) {
            lds_barrier();
            bias_to_lds<T>(a, w, head);
        }
        for (int q0 = it.k_begin; q0 < it.k_end; q0 += kRows) {
            put_stats(head, q0);
            loads_done_barrier();
            buf ^= 1;
            int next_q = q0 + kRows, next_head = head;
            if (next_q >= it.k_end) next_q = it.k_begin, ++next_head;
            const bool more = next_head < (kv_head + 1) * a.share;
            const int next_n = it.k_end - next_q, to = (buf ^ 1) * kBuf;
            // after the last step zeros are requested: a branch less among the products
            const char* const next_qs = more ? a.q.p + (int64_t)(it.q_row + next_q) * a.q.row + next_head * a.q.head : a.zeros;
            const char* const next_gs = more ? a.d_o.p + (int64_t)(it.q_row + next_q) * a.d_o.row + next_head * a.d_o.head : a.zeros;
            const int q_pitch = more ? (int)a.q.row : 0, g_pitch = more ? (int)a.d_o.row : 0;
            if (more) fetch_stats(next_head, next_q);
            // key0 counts in query rows: row i sees the keys up to its own place
            if (count == 0 || (a.causal && q0 + kRows <= key0)) {
                feed.load(next_qs, q_pitch, next_n, to);
                feed.load(next_gs, g_pitch, next_n, to + kBuf / 2);
                continue;
            }
            constexpr int kPer = RowFeed<T, D, kRows>::kEach / kTilesOf;  // requests of each of the two tensors in a tile of rows
            auto ask_q = [&](int u) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) feed.one(u * kPer + i, next_qs, q_pitch, next_n, to);
            };
            auto ask_g = [&](int u) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) feed.one(u * kPer + i, next_gs, g_pitch, next_n, to + kBuf / 2);
            };
            const char* const qs = lds + buf * kBuf;
            const char* const gs = qs + kBuf / 2;
            const float* const row_lse = stats + buf * 2 * kRows;
            const float* const row_delta = row_lse + kRows;
            const int some_large = SHAPED && a.span ? large[buf] : 0;
            // each product's fragments are requested one product ahead
            AsRows<T, D> qr;
            qr.load(qs, 32 * half, lane);
#pragma unroll
            for (int u = 0; u < kTilesOf; ++u) {
                const int row = 32 * (half + u), first = q0 + row;
                f32x16 p, ds;
                f32x4 lse[4], delta[4];
                AsRows<T, D> gr;
                AsColumns<T, D> gc, qc;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    lse[g] = *reinterpret_cast<const f32x4*>(row_lse + row + 8 * g + 4 * h);
                    delta[g] = *reinterpret_cast<const f32x4*>(row_delta + row + 8 * g + 4 * h);
                }
                phase();
                gr.load(gs, row, lane);
                qr.dot(p, k);
                woven<0, 1, 0>();
                ask_q(u);
                gc.load(gs, row, lane);
                if constexpr (SHAPED) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[i] *= scale2;
                    if (a.span) {
                        add_bias<-1>(p, a, w, key0, first, r, h);
                        if (__builtin_amdgcn_readfirstlane(some_large)) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) p[i] = fminf(p[i] - tops[buf * kRows + row + 8 * (i >> 2) + 4 * h + (i & 3)], 0.f);
                        }
                    }
                    if (a.causal && first < key0 + 31) {  // rows before `last` do not see the lane's key
                        const int last = key0 + r - first - 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[i] = 8 * (i >> 2) + (i & 3) >= last ? p[i] : kNone;
                    }
                }
                gr.dot(ds, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = weight_of<SHAPED>(p[i], scale2, lse[i >> 2][i & 3]);
                woven<0, 2, 6>();
                ask_g(u);
                qc.load(qs, row, lane);
                gc.add(dv, p);
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] = p[i] * (ds[i] - delta[i >> 2][i & 3]);
                woven<4, 2, 7>();
                if constexpr (kFine) {
                    if (fine) {
                        gc.add_rest(dv, p);
                        phase();
                    }
                }
                if (u + 1 < kTilesOf) qr.load(qs, row + 32, lane);
                qc.add(dk, ds);
                woven<4, 1, 1>();
                if constexpr (kFine) {
                    if (fine) {
                        qc.add_rest(dk, ds);
                        phase();
                    }
                }
            }
        }
    }
    loads_done_barrier();
    if (!live) {  // its weights were those of a key of zeros
        clear<R::kTiles>(dk);
        clear<R::kTiles>(dv);
    }
    char* const scratch = lds + wave * 32 * R::kPitch;
    auto put_dk = [&] { store_tile<T, D>(dk, a.scale, scratch, a.dk.p + k_row0 * a.dk.row + kv_head * a.dk.head, a.dk.row, count, lane); };
    auto put_dv = [&] { store_tile<T, D>(dv, 1.f, scratch, a.dv.p + k_row0 * a.dv.row + kv_head * a.dv.head, a.dv.row, count, lane); };
    if constexpr (!PAIR) {
        put_dk();
        put_dv();
    } else {  // of two wavefronts with the same keys the first takes the other's dK and gives it its dV
        auto at = [&](int of, int t, int g) { return reinterpret_cast<f32x4*>(lds) + (t * 4 + g) * 256 + of * 64 + lane; };
        auto give = [&](const f32x16* x) {
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) *at(wave, t, g) = f32x4{x[t][4 * g], x[t][4 * g + 1], x[t][4 * g + 2], x[t][4 * g + 3]};
        };
        auto take = [&](f32x16* x) {
#pragma unroll
            for (int t = 0; t < R::kTiles; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = *at(wave ^ 2, t, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][4 * g + e] += v[e];
                }
        };
        if (half) give(dk);
        else give(dv);
        lds_barrier();
        if (half) take(dv);
        else take(dk);
        lds_barrier();
        if (half) put_dv();
        else put_dk();
    }
}

// ---------------------------------------------------------------- launches
namespace {

size_t bias_bytes(const RaggedArgs& a) { return (a.span + 2 * kMargin) * sizeof(float); }

template <typename K> hipError_t launch(K kernel, DeviceOnce& once, int64_t blocks, size_t lds, const RaggedArgs& a, hipStream_t s) {
    hipError_t e = once.run([&] { return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - 1024); });
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)blocks), dim3(256), lds, s>>>(a);
    return hipGetLastError();
}
// f(type, head size, bias)
template <typename F> hipError_t by_kind(int head_dim, bool bf16, bool bias, F f) {
    if (bf16) {
        if (head_dim == 128) return bias ? f((bf16_t*)nullptr, std::integral_constant<int, 128>(), std::true_type()) : f((bf16_t*)nullptr, std::integral_constant<int, 128>(), std::false_type());
        return bias ? f((bf16_t*)nullptr, std::integral_constant<int, 64>(), std::true_type()) : f((bf16_t*)nullptr, std::integral_constant<int, 64>(), std::false_type());
    }
    if (head_dim == 128) return bias ? f((float*)nullptr, std::integral_constant<int, 128>(), std::true_type()) : f((float*)nullptr, std::integral_constant<int, 128>(), std::false_type());
    return bias ? f((float*)nullptr, std::integral_constant<int, 64>(), std::true_type()) : f((float*)nullptr, std::integral_constant<int, 64>(), std::false_type());
}

}  // namespace

hipError_t launch_attn_forward(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr, [&](auto* t, auto d, auto bias) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool B = decltype(bias)::value;
        typedef Rows<T, D> R;
        static DeviceOnce once_few, once_pair, once_many;
        const int64_t blocks = (int64_t)a.n_items * a.heads;
        const size_t w = B ? bias_bytes(a) : 0, lds = 2 * Steps<T, D>::kBuf + w;
        if (tile_rows == kAttnFew) return launch(attn_few_kernel<T, D, B>, once_few, blocks, 4 * 2 * 32 * R::kPitch + w, a, s);
        if constexpr (!R::kWide)
            if (tile_rows == kAttnPair) return launch(attn_forward_kernel<T, D, B, true>, once_pair, blocks, lds, a, s);
        return launch(attn_forward_kernel<T, D, B, false>, once_many, blocks, lds, a, s);
    });
}

hipError_t launch_attn_join(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, int joins, hipStream_t s) {
    if (joins == 0) return hipSuccess;
    return by_kind(head_dim, bf16, false, [&](auto* t, auto d, auto) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        attn_join_kernel<T, D><<<dim3(joins, a.heads, (tile_rows * (D / 4) + 255) / 256), 256, 0, s>>>(a, tile_rows);
        return hipGetLastError();
    });
}

hipError_t launch_attn_dq(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr, [&](auto* t, auto d, auto bias) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool B = decltype(bias)::value;
        static DeviceOnce once_pair, once_many;
        const int64_t blocks = (int64_t)a.n_items * a.heads;
        const size_t lds = 2 * Steps<T, D>::kBuf + (B ? 9 * bias_bytes(a) : 0);
        if constexpr (!Rows<T, D>::kWide)
            if (tile_rows == kAttnPair) return launch(attn_dq_kernel<T, D, B, true>, once_pair, blocks, lds, a, s);
        return launch(attn_dq_kernel<T, D, B, false>, once_many, blocks, lds, a, s);
    });
}

hipError_t launch_attn_dkv(const RaggedArgs& a, int head_dim, bool bf16, int tile_keys, hipStream_t s) {
    const int64_t blocks = (int64_t)a.n_items * (a.heads / a.share) + (a.bias ? (a.buckets * a.heads + 3) / 4 : 0);
    if (blocks == 0) return hipSuccess;
    return by_kind(head_dim, bf16, a.bias != nullptr || a.causal, [&](auto* t, auto d, auto shaped) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int D = decltype(d)::value;
        constexpr bool S = decltype(shaped)::value;
        static DeviceOnce once_pair, once_many;
        const size_t lds = 2 * Steps<T, D>::kBuf + (6 * Rows<T, D>::kStep + kLargeFlags) * sizeof(float) + (S ? bias_bytes(a) : 0);
        if constexpr (!Rows<T, D>::kWide)
            if (tile_keys == kAttnPair) return launch(attn_dkv_kernel<T, D, S, true>, once_pair, blocks, lds, a, s);
        return launch(attn_dkv_kernel<T, D, S, false>, once_many, blocks, lds, a, s);
    });
}

}  // namespace aed
