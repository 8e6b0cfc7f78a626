// The pieces that passes of cross attention are divided into, compiled for the
// host alone (no HIP function is called) with undefined behaviour trapped: none
// is shorter than the rule of dense_division.h says.  Prints "ok".
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "dense_division.h"

using namespace f3s;

int main()
{
    std::mt19937 rng(11);
    int64_t least = 1 << 30, pieces = 0;
    for (int round = 0; round < 20000; ++round) {
        const int B = 1 + (int)(rng() % 12), heads = 1 + (int)(rng() % 9);
        const int most_rows = 1 << (rng() % 13), most_others = 1 << (rng() % 14);
        std::vector<Range> ranges;
        int64_t row = 0, other = 0;
        for (int b = 0; b < B; ++b) {
            const int64_t n = 1 + rng() % most_rows, m = rng() % (most_others + 1);
            ranges.push_back({row, n, other, m});
            row += n;
            other += m;
        }
        for (int64_t slots : {128, 256, 512, 768, 1024}) {
            Division d;
            d.make(ranges, heads, slots == 1024 ? 16 : 128, 64, 256, slots);
            for (const DenseItem &i : d.items)
                if (i.part >= 0) {
                    ++pieces;
                    if (i.others < least) least = i.others;
                }
        }
    }
    if (least < 128 || pieces < 100000) {
        printf("a piece of %lld rows, %lld pieces\n", (long long)least, (long long)pieces);
        return 1;
    }
    printf("ok\n");
    return 0;
}
