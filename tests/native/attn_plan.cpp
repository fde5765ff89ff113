// The work lists of csrc/attn_plan.h over many batches: every visible pair of a row and a key in exactly one item of each list, rows and
// parts in bounds, every row written; buckets by the rule in whole numbers.
#include <stdio.h>

#include <map>
#include <set>

#include "attn_plan.h"

using namespace aed;

static int bad = 0;
static void expect(bool ok, const char* what, long long a, long long b, long long c) {
    if (!ok && bad++ < 20) printf("%s: %lld, %lld, %lld\n", what, a, b, c);
}
static unsigned seed = 1;
static unsigned rnd(unsigned n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; }

static void check(const std::vector<int32_t>& q, const std::vector<int32_t>& k, bool causal, bool starts, bool pairs, int heads, int kv_heads) {
    const int B = (int)q.size();
    std::vector<int64_t> at(B);
    int64_t packed = 0;
    for (int b = 0; b < B; ++b) {
        at[b] = starts ? 100000ll * ((b * 7) % B) + 5000000000ll : packed;
        packed += k[b];
    }
    const AttnPlan p = plan_attention(q.data(), k.data(), starts ? at.data() : nullptr, B, heads, kv_heads, causal, !starts, 128, pairs ? 64 : 0, 32);
    std::vector<int> first(B + 1, 0);
    for (int b = 0; b < B; ++b) first[b + 1] = first[b] + q[b];
    auto seq_of = [&](int row) { return (int)(std::upper_bound(first.begin(), first.end(), row) - first.begin()) - 1; };
    expect(p.q_rows == first[B], "rows", p.q_rows, first[B], 0);
    // forward and query gradients: per row, the keys that its items hold, in order and without a gap
    for (int list = 0; list < (starts ? 1 : 2); ++list) {
        const int tile = list ? p.dq_rows : p.tile_rows;
        std::map<int, std::vector<std::pair<int, int>>> held;
        std::map<int, int> parts;
        std::set<int> used;
        for (const PlanItem& it : list ? p.dq : p.forward) {
            const int b = seq_of(it.q_row), nq = q[b], nk = k[b], q0 = it.q_row - first[b];
            expect(it.rows >= 1 && it.rows <= tile && q0 % tile == 0 && q0 + it.rows <= nq, "rows of an item", it.q_row, it.rows, tile);
            expect(it.k_row == at[b] && it.pos == nk - nq + q0, "place", it.k_row, it.pos, b);
            expect(it.k_begin >= 0 && it.k_begin <= it.k_end && it.k_end <= nk, "keys of an item", it.k_begin, it.k_end, nk);
            held[it.q_row].push_back({it.k_begin, it.k_end});
            parts[it.q_row] = it.rows;
            if (it.part >= 0) expect(used.insert(it.part).second && it.part < p.n_parts, "part", it.part, p.n_parts, 0);
            else expect(held[it.q_row].size() == 1, "whole items are alone", it.q_row, 0, 0);
        }
        long long rows = 0;
        for (auto& h : held) {
            std::sort(h.second.begin(), h.second.end());
            const int b = seq_of(h.first), pos = k[b] - q[b] + h.first - first[b], need = causal ? std::max(0, std::min(k[b], pos + parts[h.first])) : k[b];
            int end = 0;
            for (auto& r : h.second) {
                expect(r.first == end, "gap or overlap", h.first, r.first, end);
                end = r.second;
            }
            expect(end == need, "keys of a row", h.first, end, need);
            rows += parts[h.first];
        }
        expect(rows == first[B], "every row once", rows, first[B], list);
        if (!list) {
            long long joined = 0;
            for (const PlanJoin& j : p.joins) {
                joined += j.n_parts;
                expect(j.n_parts >= 2 && parts[j.q_row] == j.rows && (int)held[j.q_row].size() == j.n_parts, "join", j.q_row, j.n_parts, j.rows);
                for (int i = 0; i < j.n_parts; ++i) expect(used.count(j.part + i) == 1, "joined part", j.part, i, 0);
            }
            expect(joined == p.n_parts, "parts", joined, p.n_parts, 0);
        }
    }
    if (starts) return;
    // key gradients: every key once, with all rows that see it
    std::set<int64_t> keys;
    for (const PlanItem& it : p.dkv) {
        int b = 0;
        while (!(it.k_row >= at[b] && it.k_row < at[b] + k[b])) ++b;
        const int k0 = (int)(it.k_row - at[b]);
        expect(it.rows >= 1 && it.rows <= p.dkv_keys && k0 % p.dkv_keys == 0 && k0 + it.rows <= k[b], "keys of an item", k0, it.rows, k[b]);
        expect(it.q_row == first[b] && it.k_end == q[b] && it.pos == k0 - (k[b] - q[b]), "rows of keys", it.q_row, it.k_end, it.pos);
        expect(it.k_begin >= 0 && it.k_begin <= it.k_end && (causal ? it.k_begin <= std::max(0, it.pos) : it.k_begin == 0), "first row", it.k_begin, it.pos, 0);
        for (int i = 0; i < it.rows; ++i) expect(keys.insert(it.k_row + i).second, "a key twice", it.k_row, i, 0);
    }
    expect((int64_t)keys.size() == packed, "every key", keys.size(), packed, 0);
}

int main() {
    for (int n = 0; n < 400; ++n) {
        const int B = 1 + rnd(n % 7 ? 12 : 300), top = 1 + rnd(n % 5 ? 140 : 40), long_keys = rnd(6) == 0 ? 9000 : 520;
        std::vector<int32_t> q, k;
        for (int b = 0; b < B; ++b) q.push_back(rnd(10) ? 1 + rnd(top) : 0), k.push_back(rnd(12) ? 1 + rnd(long_keys) : 0);
        const int heads = 1 << rnd(5);
        for (int c = 0; c < 8; ++c) check(q, k, c & 1, c & 2, c & 4, heads, heads >> rnd(2) ? heads >> rnd(2) : 1);
        check(q, q, true, false, true, heads, heads);
    }
    // buckets: bucket half + i begins at the first n with (n / half)^(side - half) >= (max / half)^i, in whole numbers of 128 bits
    const int rules[][2] = {{2, 2}, {3, 5}, {4, 9}, {8, 20}, {16, 64}, {32, 128}, {12, 1000}, {7, 1024}, {6, 24}, {8, 64}};
    for (auto& rule : rules)
        for (int two = 0; two < 2; ++two) {
            const int side = rule[0], max = rule[1], half = side / 2, e = side - half;
            const std::vector<uint8_t> of = bucket_places(side * (two + 1), max, two);
            expect((int)of.size() == (two ? 2 : 1) * max + 1, "places", of.size(), max, two);
            for (int d = 0; d < (int)of.size(); ++d) {
                const int n = d < max ? max - d : d - max;
                long double power = 1;  // enough for a comparison unless the two sides are near, which is looked at exactly below
                int b = n;
                if (n >= half) {
                    b = half;
                    while (b + 1 < side) {
                        const int i = b + 1 - half;
                        power = powl((long double)n / half, e) / powl((long double)max / half, i);
                        bool past = power >= 1;
                        if (fabsl(power - 1) < 1e-12L) {  // equal powers: n^e half^i = half^e max^i
                            unsigned __int128 x = 1, y = 1;
                            bool fits = true;
                            for (int j = 0; j < e; ++j) x *= n, y *= half, fits = fits && x < ((unsigned __int128)1 << 110) && y < ((unsigned __int128)1 << 110);
                            for (int j = 0; j < i; ++j) x *= half, y *= max, fits = fits && x < ((unsigned __int128)1 << 110) && y < ((unsigned __int128)1 << 110);
                            if (fits) past = x >= y;
                        }
                        if (!past) break;
                        ++b;
                    }
                }
                if (two && d > max) b += side;
                expect(of[d] == b, "bucket", side, n, of[d]);
            }
        }
    if (bad) printf("%d mistakes\n", bad);
    return bad != 0;
}
