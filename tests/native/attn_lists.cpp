// What the work lists of csrc/attn_plan.h promise beyond their completeness: the number of workgroups that an argument check counts on, which lengths
// are split, and that a split is taken only where its estimate is the shorter.
#include <stdio.h>

#include "attn_plan.h"

using namespace aed;

static unsigned seed = 7;
static unsigned rnd(unsigned n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; }

int main() {
    int bad = 0, split = 0, halves = 0, few = 0;
    auto expect = [&](bool ok, const char* what, long long a, long long b) {
        if (!ok && bad++ < 20) printf("%s: %lld, %lld\n", what, a, b);
    };
    for (int n = 0; n < 3000; ++n) {
        const int B = 1 + rnd(n % 5 ? 8 : 200), top = 1 + rnd(n % 3 ? 448 : 40), long_keys = 1 + rnd(n % 2 ? 12000 : 900), heads = 1 + rnd(16), pair = n % 4 ? 64 : 0;
        std::vector<int32_t> q, k;
        int64_t q_rows = 0, k_rows = 0;
        int most_keys = 0;
        for (int b = 0; b < B; ++b) {
            q.push_back(rnd(top + 1)), k.push_back(rnd(long_keys + 1));
            q_rows += q.back(), k_rows += k.back(), most_keys = std::max(most_keys, (int)k.back());
        }
        const AttnPlan p = plan_attention(q.data(), k.data(), nullptr, B, heads, heads, n % 7 == 0, true, 128, pair, 32, n % 3 == 0, n % 8 < 4 ? 64 : 128);
        const int64_t bound = std::max(q_rows, k_rows) / 32 + B + kPlanMost;
        for (auto* list : {&p.forward, &p.dq, &p.dkv}) expect((int64_t)list->size() <= bound, "items", list->size(), bound);
        if (p.n_parts > 0) {
            expect((int64_t)p.forward.size() * heads <= kPlanMost, "workgroups of a split list", p.forward.size(), heads);
            expect(most_keys >= kPlanLong, "split though short", most_keys, p.n_parts);
            for (const PlanItem& it : p.forward)
                if (it.part >= 0) expect(it.k_end > it.k_begin, "empty part", it.part, it.k_end);
        }
        expect(p.tile_rows == 128 || p.tile_rows == 32 || (pair && p.tile_rows == 64), "rows of an item", p.tile_rows, pair);
        split += p.n_parts > 0, halves += p.tile_rows == 64, few += p.tile_rows == 32;
    }
    // one workgroup a compute unit for as long as there are units: a split of two halves the walk, and the estimate says so
    for (int kind = 0; kind < 8; ++kind) {
        const WalkCost c = walk_cost(kind & 1, kind & 2 ? 128 : 64, kind & 4, 64);
        expect(walk_time({100}, 50, 8, c) < walk_time({100}, 100, 8, c), "one long item", kind, 0);
        expect(walk_time(std::vector<int>(64, 20), 10, 8, c) > walk_time(std::vector<int>(64, 20), 20, 8, c) || c.both == 0, "a full chip", kind, 0);
        expect(walk_time({}, 1, 8, c) == 0 && walk_time({0, 0}, 1, 8, c) > 0, "nothing to walk", kind, 0);
    }
    expect(split > 100 && halves > 100 && few > 20, "forms that occur", split, halves);
    if (bad) printf("%d mistakes\n", bad);
    return bad != 0;
}
