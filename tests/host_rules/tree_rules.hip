// Where the bits of a drafted tree are read, compiled for the host alone (no HIP function is
// called) with undefined behaviour trapped: for every tile of keys that a tree's kernels walk,
// both words lie in the row, and the bits of the keys that are there are the row's.  Prints
// "ok".
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "dense_common.h"

using namespace f3s;

#define CHECK(c)                                                           \
    do {                                                                   \
        if (!(c)) {                                                        \
            printf("check failed: %s (line %d)\n", #c, __LINE__);          \
            exit(1);                                                       \
        }                                                                  \
    } while (0)

// Token t of the tree is seen if bit t % 7 of `seen` is set; all before the tree is.
static bool sees(int seen, int token) { return token < 0 || (seen >> token % 7 & 1); }

// A draft of n tokens at the end of `len` cached ones, keys by tiles of `tile`, 32 at a time.
static void check(int n, int len, int tile, int seen)
{
    const int32_t base = (int32_t)cache_position(len, n, 0);
    std::vector<uint32_t> row(kTreeWords, 0);
    row[0] = ~0u;
    for (int t = 0; t < n; ++t)
        if (sees(seen, t)) row[t / 32 + 1] |= 1u << t % 32;
    for (int key0 = 0; key0 < len; key0 += tile)
        for (int key = key0; key < key0 + tile; key += 32) {
            const int32_t at = tree_place(key, base);
            const int32_t word = (at >> 5) + 1;
            CHECK(word >= 0 && word + 1 < kTreeWords);
            const uint64_t both = (uint64_t)row[word + 1] << 32 | row[word];
            const uint32_t bits = (uint32_t)(both >> (at & 31));
            for (int j = 0; j < 32 && key + j < len; ++j)
                CHECK((bits >> j & 1) == sees(seen, key + j - base));
        }
}

int main()
{
    for (int n = 1; n <= kTreeTokens; ++n)
        for (int len = n < 40 ? 0 : n % 64; len <= n + 70; ++len)
            for (int tile : {32, 64})
                check(n, len, tile, (n * 5 + len) % 127);
    check(kTreeTokens, 100001, 64, 77);
    // a prefix, all of which lies ahead of any tree, and the largest numbers
    CHECK(tree_place(0, 1 << 30) == -32 && tree_place((1 << 30) - 1, 1 << 30) == -1);
    CHECK(tree_place(1 << 30, -kTreeTokens) == kTreeTokens - 1);
    printf("ok\n");
    return 0;
}
