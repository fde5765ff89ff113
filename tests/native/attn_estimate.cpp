// The number of parts that csrc/attn_plan.h takes for split keys is the one whose estimate is the shortest, and shorter than that of whole items.
#include <stdio.h>

#include <map>

#include "attn_plan.h"

using namespace aed;

static unsigned seed = 11;
static unsigned rnd(unsigned n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; }

int main() {
    int bad = 0, split = 0, whole = 0, not_last = 0;
    auto expect = [&](bool ok, const char* what, double a, double b) {
        if (!ok && bad++ < 20) printf("%s: %g, %g\n", what, a, b);
    };
    for (int n = 0; n < 4000; ++n) {
        const int B = 1 + rnd(n % 5 ? 8 : 120), top = 1 + rnd(n % 3 ? 448 : 40), long_keys = 200 + rnd(n % 2 ? 12000 : 2000), heads = 1 + rnd(16), pair = n % 4 ? 64 : 0;
        const bool bf16 = n % 3 == 0;
        const int head_dim = n % 8 < 4 ? 64 : 128;
        std::vector<int32_t> q, k;
        int most = 0, most_keys = 0;
        for (int b = 0; b < B; ++b) {
            q.push_back(1 + rnd(top)), k.push_back(1 + rnd(long_keys));
            most = std::max(most, (int)q.back()), most_keys = std::max(most_keys, (int)k.back());
        }
        const AttnPlan p = plan_attention(q.data(), k.data(), nullptr, B, heads, heads, n % 7 == 0, false, 128, pair, 32, bf16, head_dim);
        // the items as they were before they were split: steps of a walk, parts taken
        const int step = p.tile_rows == 32 ? 128 : 64;
        std::map<int, std::pair<int, int>> items;
        for (const PlanItem& it : p.forward) {
            auto& of = items[it.q_row];
            of.first = std::max(of.first, it.k_end);
            of.second += 1;
        }
        std::vector<int> steps;
        for (auto& it : items) steps.push_back((it.second.first + step - 1) / step);
        const int longest = *std::max_element(steps.begin(), steps.end());
        auto fits = [&](int share) {
            size_t i = 0;
            for (auto& it : items)
                if (std::max(1, (steps[i++] + share - 1) / share) != it.second.second) return false;
            return true;
        };
        int taken = std::max(longest, 1);
        while (taken > 1 && !fits(taken)) --taken;
        expect(fits(taken), "no share has these parts", n, longest);
        if (most_keys < kPlanLong || (int64_t)items.size() * heads > kPlanMost) {
            expect(p.n_parts == 0, "split though short or many", n, p.n_parts);
            continue;
        }
        const WalkCost cost = walk_cost(bf16, head_dim, p.tile_rows == pair, most);
        const double time = walk_time(steps, taken, heads, cost), unsplit = walk_time(steps, longest, heads, cost);
        expect(p.n_parts ? time < unsplit : time == unsplit, "estimate of what was taken and of whole items", time, unsplit);
        int last = longest;
        for (int parts = 2; longest >= parts * (kPlanPart / step); ++parts) {
            const int share = (longest + parts - 1) / parts;
            int64_t all = 0;
            for (const int s : steps) all += std::max(1, (s + share - 1) / share);
            if (all * heads > kPlanMost) break;
            last = share;
            expect(walk_time(steps, share, heads, cost) >= time, "a shorter estimate was left", walk_time(steps, share, heads, cost), time);
        }
        split += p.n_parts > 0, whole += p.n_parts == 0;
        not_last += p.n_parts > 0 && !fits(last);
    }
    expect(split > 100 && whole > 100 && not_last > 100, "forms that occur", split, whole);
    if (bad) printf("%d mistakes\n", bad);
    else printf("%d split, %d of them in less than the most parts, %d whole\n", split, not_last, whole);
    return bad != 0;
}
