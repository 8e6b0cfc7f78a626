// The rules of a window of keys, compiled for the host alone (no HIP function is called)
// with undefined behaviour trapped, against plain statements of them.  Prints "ok".
#include <stdio.h>
#include <stdlib.h>

#include <random>
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

static bool sees(long w, long s, long p, long j)
{
    return j >= 0 && j <= p && (j > p - w || j < s);
}

int main()
{
    std::mt19937 rng(1);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int turn = 0; turn < 20000; ++turn) {
        const int scale = turn % 3 == 0 ? 12 : turn % 3 == 1 ? 150 : 600;
        const WindowRule w = {turn % 17 ? pick(0, scale) : 1 << 30, pick(0, scale / 2)};
        const int first = pick(-5, scale), last = first + pick(0, 130);
        const int key = pick(0, scale), n = pick(1, 64);
        bool all = true, none = true;
        for (int p = first; p <= last; ++p)
            for (int j = key; j < key + n; ++j) {
                const bool s = sees(w.window, w.sinks, p, j);
                CHECK(window_sees(w, p, j) == s);
                all = all && s;
                none = none && !s;
            }
        // each may be missed, but never claimed wrongly; and neither is missed where it
        // would cost most: whole tiles of the middle of a window, tiles outside it
        CHECK(!window_all(w, first, last, key, n) || all);
        CHECK(!window_none(w, first, last, key, n) || none);
        if (key >= w.sinks) {
            CHECK(window_all(w, first, last, key, n) == all);
            CHECK(window_none(w, first, last, key, n) == none || w.window == 0);
        }

        const int step = turn & 1 ? 1 : 16;
        const WindowKeys k = window_keys(w, first, last, step);
        const int length = window_length(k);
        CHECK(length >= 0 && k.near % step == 0);
        if (last < 0) {
            CHECK(length == 0);
            continue;
        }
        std::vector<int> times(last + 1, 0);
        for (int tile : {32, 64})
            for (int v = 0; v < length; v += tile) {
                const KeyRun r = window_run(k, v);
                // a tile lies in one of the two parts, and every key that it would load
                // is there
                CHECK(r.key >= 0 && r.key <= last && r.key % step == 0);
                for (int i = 0; i < tile && i < r.left; ++i) {
                    CHECK(r.key + i <= last);
                    if (tile == 64) ++times[r.key + i];
                }
            }
        for (int j = 0; j <= last; ++j) {
            CHECK(times[j] <= 1);
            if (times[j]) continue;
            for (int p = first < 0 ? 0 : first; p <= last; ++p)
                CHECK(!sees(w.window, w.sinks, p, j));
        }
        // what is walked beside the keys that are seen is bounded
        if (w.window < (1 << 29))
            CHECK(length <= w.window + w.sinks + (last - first) + 2 * 64 + 2 * step);
    }
    // the largest numbers
    const WindowRule most = {1 << 30, 0};
    CHECK(window_sees(most, 0x7FFFF000, 0x7FFFF000 - (1 << 30) + 1));
    CHECK(!window_sees(most, 0x7FFFF000, 0x7FFFF000 - (1 << 30)));
    CHECK(window_keys({5, 3}, 0x7FFFEF00, 0x7FFFEF7F, 1).near == 0x7FFFEF00 - 4);
    CHECK(window_keys({1 << 30, 0}, 0x7FFFEF00, 0x7FFFEF7F, 16).near ==
          (0x7FFFEF00 - (1 << 30) + 1) / 16 * 16);
    printf("ok\n");
    return 0;
}
