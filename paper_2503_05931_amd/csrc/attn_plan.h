// Work lists of ragged attention and the buckets of its bias.  Host code without any GPU call.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <vector>

namespace aed {

// Lists are made for the whole chip: two workgroups on each of 256 compute units.
constexpr int kPlanSlots = 512;
constexpr int kPlanLong = 1024;  // keys from which on a row's may be split
constexpr int kPlanPart = 256;   // keys of a part at the least
constexpr int kPlanMost = 4 * kPlanSlots;  // workgroups up to which splitting is looked at
constexpr int64_t kPlanGrid = 0xffffffffll / 256;  // workgroups of 256 that a launch may have: its threads are counted in 32 bits

// First distances of a side's logarithmic buckets, half + 1 on: the smallest n with (n / half)^(side - half) >= (max / half)^i.
// The power is irrational but where it is a whole number, which rounding must not miss.
inline std::vector<int> bucket_steps(int side, int max_distance) {
    const int half = side / 2, log_buckets = side - half;
    std::vector<int> steps;
    for (int i = 1; i < log_buckets; ++i) {
        const double x = half * std::pow((double)max_distance / half, (double)i / log_buckets), whole = std::nearbyint(x);
        steps.push_back((int)(std::fabs(x - whole) < 1e-11 * whole ? whole : std::ceil(x)));
    }
    return steps;
}
// Bucket by place = key - query + max_distance; max_distance + 1 places, with bidirectional buckets 2 max_distance + 1
inline std::vector<uint8_t> bucket_places(int buckets, int max_distance, bool bidirectional) {
    const int side = bidirectional ? buckets / 2 : buckets, half = side / 2;
    const std::vector<int> steps = bucket_steps(side, max_distance);
    std::vector<uint8_t> of;
    for (int at = 0; at <= (bidirectional ? 2 : 1) * max_distance; ++at) {
        const int n = std::abs(at - max_distance);
        int b = n;
        if (n >= half) b = half + (int)(std::upper_bound(steps.begin(), steps.end(), n) - steps.begin());
        of.push_back((uint8_t)(b + (at > max_distance ? side : 0)));
    }
    return of;
}

// Whether two of rows x heads vectors of `length` elements, `row` and `head` elements apart, share one.  Strides are not negative, and rows x row and
// heads x head below 2^62.
inline bool vectors_overlap(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t length) {
    if ((rows > 1 && row < length) || (heads > 1 && head < length)) return true;
    if (rows <= 1 || heads <= 1 || row >= (heads - 1) * head + length || head >= (rows - 1) * row + length) return false;  // one inside the other's gaps
    for (int64_t h = 1; h < heads; ++h)  // the rows whose first vectors are next to head h of row 0
        for (int64_t r = h * head / row; r <= h * head / row + 1; ++r)
            if (r >= 1 && r < rows && std::abs(r * row - h * head) < length) return true;
    return false;
}

struct PlanItem {  // RaggedItem's fields
    int64_t k_row;
    int32_t q_row, rows, pos, k_begin, k_end, part;
};
struct PlanJoin {
    int32_t q_row, rows, part, n_parts;
};

// Microseconds of the forward kernel: a step of a workgroup alone on its compute unit, how many times as long it takes if two are there (0: two do
// not fit), a part and head of the join.  Rows shared in pairs: a wavefront has half of a step's keys, and if there are 32 rows at the most, half of the
// wavefronts have none, which float32 products leave to the others.
struct WalkCost {
    double step, both, part;
};
inline WalkCost walk_cost(bool bf16, int head_dim, bool pairs, int most_rows) {
    const WalkCost c = bf16 ? (head_dim == 128 ? WalkCost{1.85, 1.6, 0.016} : WalkCost{1.15, 1.35, 0.008})
                            : (head_dim == 128 ? WalkCost{10.3, 0.0, 0.016} : WalkCost{5.0, pairs && most_rows <= 32 ? 1.1 : 1.9, 0.008});
    return WalkCost{pairs ? 0.6 * c.step : c.step, c.both, c.part};
}
// and over items of `steps` steps each, split into parts of at most `share`, longest first: rounds of workgroups, 5 us to start each, 2 us for the
// join's launch.  Measured on 12 batches of 1 to 40 sequences, 1 to 448 rows and 1000 to 8000 keys, 0 to 24 parts each (8 heads of 128 in bfloat16, and
// 6 of them in the other kinds): what this finds best takes at most 12 % longer than what was.  (Part counts by the chip's share alone,
// three workgroups to two slots: up to 30 % longer, as most of the last round of workgroups was idle.)
inline double walk_time(const std::vector<int>& steps, int64_t share, int heads, const WalkCost& cost) {
    int64_t items = 0, parts = 0, longest = 0, total = 0;
    for (const int n : steps) {
        const int64_t of = std::max<int64_t>(1, (n + share - 1) / share);
        items += of;
        total += n;
        if (of > 1) parts += of;
        longest = std::max<int64_t>(longest, (n + of - 1) / of);
    }
    if (items == 0) return 0;
    const int64_t units = kPlanSlots / 2, round = cost.both > 0 ? 2 * units : units, full = items * heads / round, left = items * heads % round;
    const double both = cost.both > 0 ? cost.both : 1.0, rounds = (double)full * both + (left == 0 ? 0 : left <= units ? 1.0 : both);
    const double mean = full > 0 ? (double)total / (double)items : (double)longest;
    return std::max(rounds * mean, (double)longest) * cost.step + 5.0 * (double)(full + (left > 0)) + (parts > 0 ? 2.0 + cost.part * (double)(parts * heads) : 0.0);
}

struct AttnPlan {
    int tile_rows = 0, dq_rows = 0, dkv_keys = 0, n_parts = 0;  // query rows of an item, forward and backward; keys of one of key gradients
    std::vector<PlanItem> forward, dq, dkv;
    std::vector<PlanJoin> joins;
    int64_t q_rows = 0;
    int64_t forward_groups = 0, dq_groups = 0, dkv_groups = 0;  // workgroups of unsplit lists; above kPlanGrid in any of them there are no lists
};

// tile_many, tile_pair (0: there are none), tile_few: query rows of an item, tile_many and tile_pair also keys of one of key gradients
inline AttnPlan plan_attention(const int32_t* q_lens, const int32_t* k_lens, const int64_t* k_starts, int batch, int heads, int kv_heads, bool causal, bool training,
                               int tile_many, int tile_pair, int tile_few, bool bf16 = true, int head_dim = 128) {
    AttnPlan p;
    int most = 0, most_keys = 0;
    int64_t by_rows = 0, by_keys = 0;
    for (int b = 0; b < batch; ++b) {
        by_rows += (q_lens[b] + tile_many - 1) / tile_many;
        by_keys += (k_lens[b] + tile_many - 1) / tile_many;
        most = std::max(most, (int)q_lens[b]);
        most_keys = std::max(most_keys, (int)k_lens[b]);
    }
    // Items of half the rows (keys), with two wavefronts to 32 of them, where twice as many workgroups still find a compute unit each, and
    // for rows where no sequence has more.  Heads of 128 in bfloat16, 120 rows and keys a sequence, forward / dQ / dK and dV in us: 128 whole items 11.4 /
    // 13.4 / 13.4, halves 10.4 / 12.5 / 13.2; 136 whole items 11.4 / 13.5 / 13.6, halves 11.7 / 16.0 / 20.6.  64 sequences of 64 rows
    // and 300 keys, whole 22.8 / 27.1, halves 21.5 / 26.8; of 120 rows and 64 keys, dK and dV whole 24.9, halves 26.2.
    const bool few_rows = by_rows * heads <= kPlanSlots / 4, few_keys = by_keys * kv_heads <= kPlanSlots / 4;
    p.dq_rows = tile_pair && (most <= tile_pair || few_rows) ? tile_pair : tile_many;
    p.dkv_keys = tile_pair && few_keys ? tile_pair : tile_many;
    // Forward, up to 16 rows (up to all 32 where there are no halves) have a kernel of their own, unless keys are split: 256 sequences of 124 keys,
    // 1 / 16 / 32 rows, 28.6 / 34.0 / 42.3 us, halves 30.7 / 34.2 / 36.4; 8 of 500 keys, 1 / 32 rows, 11.3 / 13.6, halves 13.9 / 14.4; 5 of 4000
    // keys, 1 / 16 / 32 rows, 19.9 / 21.8 / 24.8, halves 18.3 / 18.9 / 19.2.  Where keys are split there are items enough without
    // halves: 14 items of 128 rows against 2000 to 6000 keys take 79 us so, 89 us in halves.
    const bool split = most_keys >= kPlanLong;
    if (tile_pair ? most <= tile_few / 2 && !split : most <= tile_few) p.tile_rows = tile_few;
    else p.tile_rows = split && most > tile_pair ? tile_many : p.dq_rows;
    auto count = [&](const int32_t* lens, int tile) {
        int64_t n = 0;
        for (int b = 0; b < batch; ++b) n += (lens[b] + (int64_t)tile - 1) / tile;
        return n;
    };
    p.forward_groups = count(q_lens, p.tile_rows) * heads;
    if (training) p.dq_groups = count(q_lens, p.dq_rows) * heads, p.dkv_groups = count(k_lens, p.dkv_keys) * kv_heads;
    if (std::max(p.forward_groups, std::max(p.dq_groups, p.dkv_groups)) > kPlanGrid) return p;
    const int step = p.tile_rows == tile_few ? 128 : 64;  // keys that a workgroup takes at once
    std::vector<PlanItem> whole;
    int64_t q_row = 0, packed = 0;
    auto tiles = [&](int tile, std::vector<PlanItem>& to, int b, int64_t k_row) {
        const int nq = q_lens[b], nk = k_lens[b];
        for (int q0 = 0; q0 < nq; q0 += tile) {
            const int rows = std::min(tile, nq - q0), pos = nk - nq + q0;
            to.push_back(PlanItem{k_row, (int32_t)(q_row + q0), rows, pos, 0, causal ? std::max(0, std::min(nk, pos + rows)) : nk, -1});
        }
    };
    for (int b = 0; b < batch; ++b) {
        const int nq = q_lens[b], nk = k_lens[b];
        const int64_t k_row = k_starts ? k_starts[b] : packed;
        tiles(p.tile_rows, whole, b, k_row);
        if (training) {
            tiles(p.dq_rows, p.dq, b, k_row);
            for (int k0 = 0; k0 < nk; k0 += p.dkv_keys) {
                const int pos = k0 - (nk - nq);
                p.dkv.push_back(PlanItem{k_row + k0, (int32_t)q_row, std::min(p.dkv_keys, nk - k0), pos, causal ? std::max(0, std::min(nq, pos)) : 0, nq, -1});
            }
        }
        q_row += nq;
        packed += nk;
    }
    p.q_rows = q_row;
    std::vector<int> steps;
    for (const PlanItem& it : whole) steps.push_back((it.k_end + step - 1) / step);
    const int64_t longest = steps.empty() ? 0 : *std::max_element(steps.begin(), steps.end());
    int64_t share = std::max<int64_t>(longest, 1);
    if (split && (int64_t)whole.size() * heads <= kPlanMost) {
        const WalkCost cost = walk_cost(bf16, head_dim, p.tile_rows == tile_pair, most);
        double best = walk_time(steps, share, heads, cost);
        for (int64_t parts = 2; longest >= parts * (kPlanPart / step); ++parts) {
            const int64_t with = (longest + parts - 1) / parts;
            int64_t items = 0;
            for (const int n : steps) items += std::max<int64_t>(1, (n + with - 1) / with);
            if (items * heads > kPlanMost) break;
            const double time = walk_time(steps, with, heads, cost);
            if (time < best) best = time, share = with;
        }
    }
    for (const PlanItem& it : whole) {
        const int n = (it.k_end + step - 1) / step;
        if (n <= share) {
            p.forward.push_back(it);
            continue;
        }
        const int parts = (int)((n + share - 1) / share);
        p.joins.push_back(PlanJoin{it.q_row, it.rows, p.n_parts, parts});
        for (int i = 0; i < parts; ++i) {
            PlanItem part = it;
            part.k_begin = (int)((int64_t)n * i / parts) * step;
            part.k_end = std::min(it.k_end, (int)((int64_t)n * (i + 1) / parts) * step);
            part.part = p.n_parts++;
            p.forward.push_back(part);
        }
    }
    // the longest first: they end together
    auto longer = [](const PlanItem& a, const PlanItem& b) { return a.k_end - a.k_begin > b.k_end - b.k_begin; };
    for (auto* list : {&p.forward, &p.dq, &p.dkv}) std::stable_sort(list->begin(), list->end(), longer);
    return p;
}

}  // namespace aed
