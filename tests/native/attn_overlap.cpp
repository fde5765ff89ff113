// vectors_overlap of csrc/attn_plan.h against every element of both.
#include <stdio.h>

#include <set>

#include "attn_plan.h"

int main() {
    int bad = 0, yes = 0, woven = 0;
    for (int rows = 1; rows <= 5; ++rows)
        for (int heads = 1; heads <= 5; ++heads)
            for (int row = 0; row <= 26; ++row)
                for (int head = 0; head <= 26; ++head) {
                    const int length = 4;
                    std::set<int> used;
                    for (int r = 0; r < rows; ++r)
                        for (int h = 0; h < heads; ++h)
                            for (int c = 0; c < length; ++c) used.insert(r * row + h * head + c);
                    const bool want = (int)used.size() < rows * heads * length, got = aed::vectors_overlap(rows, row, heads, head, length);
                    if (want != got && bad++ < 20) printf("%d rows by %d, %d heads by %d: %d\n", rows, row, heads, head, got);
                    yes += want;
                    woven += !want && rows > 1 && heads > 1 && row < (heads - 1) * head + length && head < (rows - 1) * row + length;
                }
    // strides at their limits: nothing overflows
    if (aed::vectors_overlap((1ll << 31) - 1, 128, 65535, 1ll << 38, 128) || !aed::vectors_overlap((1ll << 31) - 1, 1ll << 22, 65535, 1ll << 38, 128) ||
        !aed::vectors_overlap((1ll << 31) - 1, 128, 65535, 1ll << 37, 128)) bad++, printf("limits\n");
    if (!yes || !woven) bad++, printf("no such cases\n");
    return bad != 0;
}
