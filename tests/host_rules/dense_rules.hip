// The dense operators' host-side rules, compiled for the host alone (no HIP
// function is called) with undefined behaviour trapped: the division of a
// ragged batch among workgroups, the division of cached keys, places and
// powers of the cache, and the rows of a key head.  Prints "ok".
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <cmath>
#include <map>
#include <random>
#include <tuple>

#include "attend.h"
#include "dense_division.h"

using namespace f3s;

#define CHECK(c)                                                           \
    do {                                                                   \
        if (!(c)) {                                                        \
            printf("check failed: %s (line %d)\n", #c, __LINE__);          \
            exit(1);                                                       \
        }                                                                  \
    } while (0)

// Every tile of rows of every head is there, and with it every row of the other
// side exactly once, in order; partial rows are disjoint and joined by exactly
// one merge in the order of the pieces.
static void check_division(const Division &d, const std::vector<Range> &ranges, int heads,
                           int64_t tile, int64_t unit)
{
    typedef std::tuple<int, int, int> Key;  // head, row, first row of the other side's range
    std::map<Key, std::vector<DenseItem>> by;
    for (const DenseItem &i : d.items) {
        int64_t base = -1;
        for (const Range &r : ranges)
            if (i.row >= r.row && i.row < r.row + r.rows) {
                base = r.other;
                CHECK((i.row - r.row) % tile == 0);
                CHECK(i.rows == (r.row + r.rows - i.row < tile ? r.row + r.rows - i.row : tile));
                CHECK(i.other >= r.other && i.others >= 0);
                CHECK((int64_t)i.other + i.others <= r.other + r.others);
            }
        CHECK(base >= 0 && i.head >= 0 && i.head < heads);
        by[Key(i.head, i.row, (int)base)].push_back(i);
    }
    size_t tiles = 0, split = 0;
    std::map<int, int> parts;  // first partial row -> rows
    for (const Range &r : ranges)
        for (int h = 0; h < heads; ++h)
            for (int64_t at = 0; at < r.rows; at += tile) {
                ++tiles;
                auto f = by.find(Key(h, (int)(r.row + at), (int)r.other));
                CHECK(f != by.end());
                std::vector<DenseItem> v = f->second;
                std::sort(v.begin(), v.end(), [](const DenseItem &a, const DenseItem &b) {
                    return a.piece < b.piece;
                });
                int64_t next = r.other;
                for (size_t k = 0; k < v.size(); ++k) {
                    CHECK(v[k].piece == (int)k && v[k].other == next);
                    CHECK((v[k].part >= 0) == (v.size() > 1));
                    CHECK(v.size() == 1 || v[k].others > 0);
                    CHECK(v[k].others % unit == 0 || k + 1 == v.size());
                    if (v.size() > 1) {
                        CHECK(v[k].part == v[0].part + (int)k * v[0].rows);
                        CHECK(!parts.count(v[k].part));
                        parts[v[k].part] = v[k].rows;
                    }
                    next += v[k].others;
                }
                CHECK(next == r.other + r.others);
                if (v.size() > 1) {
                    int found = 0;
                    for (const DenseMerge &m : d.merges)
                        if (m.part == v[0].part) {
                            ++found;
                            CHECK(m.head == h && m.row == v[0].row && m.rows == v[0].rows);
                            CHECK(m.count == (int)v.size() && m.stride == m.rows);
                            CHECK(m.rows <= d.merge_rows);
                        }
                    CHECK(found == 1);
                    ++split;
                }
            }
    CHECK(by.size() == tiles && d.merges.size() == split);
    int64_t end = 0;
    for (const auto &p : parts) {
        CHECK(p.first == end);
        end += p.second;
    }
    CHECK(end == d.parts);
}

static void divisions()
{
    std::mt19937 rng(5);
    for (int round = 0; round < 3000; ++round) {
        const int B = (int)(rng() % 12), heads = 1 + (int)(rng() % 9);
        const int most_rows = 1 << (rng() % 13), most_others = 1 << (rng() % 14);
        std::vector<Range> ranges;
        int64_t row = 0, other = 1;
        for (int b = 0; b < B; ++b) {
            const int64_t n = 1 + rng() % most_rows, m = rng() % 8 ? rng() % (most_others + 1) : 0;
            ranges.push_back({row, n, other, m});
            row += n + rng() % 3;
            other += m + 1;
        }
        Division a, e;
        a.make(ranges, heads, 16, 64, 256, 1024);
        check_division(a, ranges, heads, 16, 64);
        const int64_t slots = 256 << (rng() % 3);
        e.make(ranges, heads, 128, 64, 256, slots);
        check_division(e, ranges, heads, 128, 64);
        for (const DenseItem &i : e.items)
            if (i.part >= 0) CHECK(i.others >= 64);
    }
    // 260 tiles on 512 places: not 520 halves (two rounds), but 512, and the four
    // behind them in short pieces
    Division d;
    d.make({{0, 4001, 0, 4095}, {4001, 4099, 4095, 4001}}, 4, 128, 64, 256, 512);
    int64_t longest = 0, whole = 0;
    for (const DenseItem &i : d.items) {
        if (i.others > longest) longest = i.others;
        whole += i.rows == 128;
    }
    check_division(d, {{0, 4001, 0, 4095}, {4001, 4099, 4095, 4001}}, 4, 128, 64);
    CHECK(whole <= 512 || longest <= 1600);
    // where all rounds are full but for a few, nothing is gained
    Division g;
    g.make({{0, 128 * 100 + 5, 0, 4096}}, 8, 128, 64, 256, 512);
    check_division(g, {{0, 128 * 100 + 5, 0, 4096}}, 8, 128, 64);
    // a few long tiles of different lengths: divided, however short the others are
    Division f;
    f.make({{0, 59, 0, 1016}, {59, 40, 1016, 760}, {99, 20, 1776, 512}}, 2, 128, 64, 256, 512);
    CHECK(f.items.size() > 15 && f.merges.size() == 6);
}

static void own_keys()
{
    std::mt19937 rng(6);
    for (int round = 0; round < 20000; ++round) {
        const int B = 1 + (int)(rng() % 40), share = 1 + (int)(rng() % 1200);
        std::vector<int32_t> units(B);
        int64_t total = 0, items = 0;
        for (auto &u : units) {
            u = units_of(rng() % 3 ? (int32_t)(rng() % 70000) : (int32_t)(rng() % 3));
            total += u;
        }
        const int32_t per = units_per_item(total, share);
        CHECK(per >= kLeastUnits);
        for (int32_t u : units) {
            const int32_t n = items_of(u, per);
            CHECK(n >= 1 && (u == 0 || n <= u));
            for (int32_t k = 0; k < n; ++k) {
                CHECK(item_unit(u, k, n) <= item_unit(u, k + 1, n));
                CHECK(item_unit(u, k + 1, n) - item_unit(u, k, n) <= per);
            }
            CHECK(item_unit(u, 0, n) == 0 && item_unit(u, n, n) == u);
            items += n;
        }
        CHECK(items <= share + B);  // the grid, and the room for partial results
    }
    CHECK(units_of(0) == 0 && units_of(1) == 1 && units_of(64) == 1 && units_of(65) == 2);
    CHECK(units_of(2147483647) == 33554432);
}

static void cache_places()
{
    const int32_t table[4] = {3, -1, 7, 0};
    for (int shift = 4; shift <= 8; ++shift) {
        const int64_t size = 1 << shift;
        CHECK(cache_slot(table, 4, 7, shift, -1) == -1);
        CHECK(cache_slot(table, 4, 7, shift, 0) == 3 * size);
        CHECK(cache_slot(table, 4, 7, shift, size - 1) == 4 * size - 1);
        CHECK(cache_slot(table, 4, 7, shift, size) == -1);          // no page
        CHECK(cache_slot(table, 4, 7, shift, 2 * size) == -1);      // behind the last page
        CHECK(cache_slot(table, 4, 8, shift, 2 * size) == 7 * size);
        CHECK(cache_slot(table, 4, 7, shift, 3 * size + 5) == 5);
        CHECK(cache_slot(table, 4, 7, shift, 4 * size) == -1);      // behind the table
        CHECK(cache_slot(table, 0, 7, shift, 0) == -1);
        CHECK(cache_slot(table, 4, 7, shift, 1ll << 40) == -1);
        const int32_t far[1] = {2147483646};
        CHECK(cache_slot(far, 1, 2147483647, shift, 3) == (2147483646ll << shift) + 3);
    }
    CHECK(cache_keys(-5, 100) == 0 && cache_keys(-2147483647 - 1, 100) == 0);
    CHECK(cache_keys(99, 100) == 99 && cache_keys(101, 100) == 100);
    CHECK(cache_keys(2147483647, 0) == 0);
    CHECK(cache_position(5, 7, 0) == -2 && cache_position(-9, 3, 2) == -1);
    CHECK(cache_position(2147483647, 1, 0) == 2147483646);
}

static void cache_powers()
{
    std::mt19937 rng(7);
    for (int k = 0; k < 2000000; ++k) {
        const uint32_t bits = k < 4096 ? (uint32_t)k << 19 & 0x7FFFFFFFu : rng() & 0x7FFFFFFFu;
        const float m = __builtin_bit_cast(float, bits);
        if (!(m <= 3.4028234664e38f)) continue;
        const int e = (int)cache_exponent(m) - 127;
        CHECK(e >= -127 && e <= 127);
        CHECK((double)m <= 448.0 * ldexp(1.0, e));
        CHECK(e == -127 || (double)m > 448.0 * ldexp(1.0, e - 1));
    }
}

static void head_rows()
{
    std::mt19937 rng(8);
    for (int g = 1; g <= 700; ++g) {
        const QueryRows q = query_rows(3 * g, g);
        for (int k = 0; k < 2000; ++k) {
            const uint32_t r = k < 3 ? 0x7FFFFFFFu - (uint32_t)k : k < 1000 ? (uint32_t)k
                                                                            : rng() >> 1;
            CHECK(row_token(q, r) == r / (uint32_t)g);
            const uint32_t edge = r / (uint32_t)g * (uint32_t)g;
            CHECK(row_token(q, edge) == edge / (uint32_t)g);
            if (edge) CHECK(row_token(q, edge - 1) == (edge - 1) / (uint32_t)g);
        }
    }
}

int main()
{
    divisions();
    own_keys();
    cache_places();
    cache_powers();
    head_rows();
    printf("ok\n");
    return 0;
}
