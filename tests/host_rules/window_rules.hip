// The rules of a window of keys, compiled for the host alone (no HIP function is called)
// with undefined behaviour trapped, against plain statements of them.  Prints "ok".
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "window_ranges.h"

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

// The items of a division: of every row of every head and every row of the other side that
// it has to meet (a query that sees a key), exactly one item has both.
static void check_plan(const std::vector<int32_t> &q_ptr, const std::vector<int32_t> &k_ptr,
                       const std::vector<int32_t> &ql, const std::vector<int32_t> &kl, int g,
                       const WindowRule &rule)
{
    const int n = (int)ql.size();
    const WindowRanges r =
        window_ranges(q_ptr.data(), k_ptr.data(), ql.data(), kl.data(), n, g, rule);
    const int64_t rows = (int64_t)q_ptr[n] * g, keys = k_ptr[n];
    std::vector<int> met(rows * keys, 0), met2(rows * keys, 0), out(rows, 0), out2(keys, 0);
    Division f, d;
    f.make(r.queries, 1, kWindowTile, kWindowUnit, 256, 64);
    d.make(r.keys, 1, kWindowTile, 64, 256, 64, Division::kLaunch, true);
    for (const DenseItem &it : f.items) {
        const WindowShared &s = r.shared[it.tag];
        CHECK(it.row >= 0 && it.rows >= 1 && it.row + it.rows <= rows);
        CHECK(it.others == 0 || it.other % kWindowUnit == 0);
        for (int i = 0; i < it.rows; ++i) out[it.row + i] += it.piece == 0;
        for (int v = 0; v < it.others; v += 64) {
            const KeyRun run = window_run(s.keys, it.other + v);
            CHECK(s.key0 + run.key >= 0 && s.key0 + run.key < keys);
            for (int j = 0; j < 64 && j < run.left; ++j) {
                CHECK(s.key0 + run.key + j < keys);
                for (int i = 0; i < it.rows; ++i)
                    ++met[(int64_t)(it.row + i) * keys + s.key0 + run.key + j];
            }
        }
    }
    for (const DenseItem &it : d.items) {
        CHECK(it.row >= 0 && it.rows >= 1 && it.row + it.rows <= keys);
        CHECK(it.others == 0 || (it.other >= 0 && it.other + it.others <= rows));
        for (int i = 0; i < it.rows; ++i) {
            out2[it.row + i] += it.piece == 0;
            for (int j = 0; j < it.others; ++j)
                ++met2[(int64_t)(it.other + j) * keys + it.row + i];
        }
    }
    for (int x : out) CHECK(x == 1);
    for (int x : out2) CHECK(x == 1);
    for (int b = 0; b < n; ++b)
        for (int64_t t = q_ptr[b]; t < q_ptr[b + 1]; ++t)
            for (int h = 0; h < g; ++h)
                for (int64_t j = 0; j < keys; ++j) {
                    const bool real = t - q_ptr[b] < ql[b] && j >= k_ptr[b] &&
                                      j < k_ptr[b] + kl[b];
                    const int64_t p = kl[b] - ql[b] + t - q_ptr[b];
                    const int64_t at = (t * g + h) * keys + j;
                    CHECK(met[at] <= 1 && met2[at] <= 1);
                    if (!real) CHECK(met[at] == 0 && met2[at] == 0);
                    if (real && sees(rule.window, rule.sinks, p, j - k_ptr[b]))
                        CHECK(met[at] == 1 && met2[at] == 1);
                }
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
    for (int turn = 0; turn < 150; ++turn) {
        const int n = pick(1, 4), top = turn % 5 ? 90 : 500, g = pick(1, 5);
        std::vector<int32_t> q = {0}, k = {0}, ql, kl;
        for (int b = 0; b < n; ++b) {
            kl.push_back(pick(0, top));
            ql.push_back(turn % 3 ? std::min(kl.back(), pick(0, top)) : pick(0, top));
            q.push_back(q.back() + ql.back() + (turn % 2 ? pick(0, 150) : 0));
            k.push_back(k.back() + kl.back() + (turn % 2 ? pick(0, 150) : 0));
        }
        check_plan(q, k, ql, kl, g,
                   {turn % 7 ? pick(0, top) : 1 << 30, turn % 4 ? pick(0, 150) : 0});
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
