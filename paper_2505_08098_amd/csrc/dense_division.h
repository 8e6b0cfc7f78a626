// How the passes of cross attention over a ragged batch are divided among
// workgroups (host only).
#pragma once

#include <algorithm>
#include <vector>

#include "dense_common.h"

namespace f3s {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One side of a pass: the rows that get results, in ranges of one sequence,
// each with the rows of the other side that it walks.
struct Range {
    int64_t row, rows, other, others;
    int32_t tag = 0;  // the caller's, handed on to its items
};

// A pass divided among workgroups, one to an item: a tile of rows of one head
// with the rows of the other side that it walks, whole or in pieces whose
// partial results are joined by merges.
struct Division {
    std::vector<DenseItem> items;  // in launch order
    std::vector<DenseMerge> merges;
    int64_t parts = 0;
    int32_t merge_rows = 0;

    // What dividing into pieces of at most `per` units takes, in units of a
    // workgroup's time, where `slots` workgroups run at once.  Pieces of nearly
    // one size run in rounds (520 on 512 places take as long as 1,024); of
    // different sizes, the longest first, they end about one piece apart.
    static double time(const std::vector<Range> &ranges, int32_t heads, int64_t tile,
                       int64_t unit, int64_t slots, int64_t per, double launch)
    {
        double total = 0, n = 0, longest = 0;
        for (const Range &r : ranges) {
            const int64_t units = ceil_div(r.others, unit), k = pieces(units, per);
            const double tiles = (double)ceil_div(r.rows, tile) * heads;
            const double one = (double)ceil_div(units, k) + (k > 1 ? kOver + kJoin : kOver);
            n += tiles * k;
            total += tiles * k * one;
            longest = one > longest ? one : longest;
        }
        const double rounds = (double)ceil_div((int64_t)n, slots);
        const double t = rounds <= 1                  ? longest
                         : longest * n <= 1.25 * total ? rounds * longest
                                                       : total / slots + longest / 2;
        return t + (split(ranges, unit, per) ? launch : 0.0);
    }
    static bool split(const std::vector<Range> &ranges, int64_t unit, int64_t per)
    {
        for (const Range &r : ranges)
            if (ceil_div(r.others, unit) > per) return true;
        return false;
    }
    static int64_t pieces(int64_t units, int64_t per)
    {
        return units <= per ? 1 : ceil_div(units, per);
    }
    static constexpr double kOver = 2;  // an item's beginning and end, in units
    static constexpr double kJoin = 1;  // a piece's partial results
    // Adding one more partial result of a row, in units (128 of them: 19 us).
    static constexpr double kPartSum = 0.07;
    // The launch that joins them, 5 us, where a unit takes 1.1 (f16, d = 64).
    static constexpr double kLaunch = 5;
    static constexpr int64_t kMostPieces = 16;
    // Times that a division by a second rule has to beat the first's (they are
    // estimates).
    static constexpr double kWorth = 0.95;
    // Tiles of a pass; a batch of more is refused.
    static constexpr double kMostTiles = 1 << 23;

    // Units of a piece, where all are divided alike, that take the least time.
    static int64_t best_pieces(const std::vector<Range> &ranges, int32_t heads, int64_t tile,
                               int64_t unit, int64_t least, int64_t slots, double launch,
                               double *takes)
    {
        const int64_t top = ranges.empty() ? 1 : ceil_div(ranges[0].others, unit);
        int64_t per = top < 1 ? 1 : top;
        double best = time(ranges, heads, tile, unit, slots, per, launch);
        for (int64_t k = 2; k <= top; k += k > kMostPieces ? k / kMostPieces : 1) {
            // (as many pieces as it takes to fill the GPU, and then some)
            const int64_t p = ceil_div(top, k);
            if (p * unit < least) break;
            const double t = time(ranges, heads, tile, unit, slots, p, launch);
            if (t < best) {
                best = t;
                per = p;
            }
            if (k > kMostPieces && k * heads > 4 * slots) break;
        }
        *takes = best;
        return per;
    }

    // Units of a piece of `rest` that take the least time, from `least` on: rounds of
    // pieces, and the adding of a row's partial results one behind the other.
    static int64_t best_rest(const std::vector<Range> &rest, int32_t heads, int64_t unit,
                             int64_t least, int64_t slots)
    {
        int64_t best = least;
        double takes = 0;
        for (int64_t s = least; s <= 16 * least; s *= 2) {
            double n = 0, most = 0;
            for (const Range &r : rest) {
                const double k = (double)pieces(ceil_div(r.others, unit), s);
                n += k * heads;
                most = k > most ? k : most;
            }
            const double t = (double)ceil_div((int64_t)n, slots) * (double)(s + kOver + kJoin) +
                             kPartSum * most;
            if (s == least || t < takes) {
                takes = t;
                best = s;
            }
        }
        return best;
    }

    // `slots`: workgroups that run at once.  A range is divided evenly into the fewest
    // pieces of at most so many units, those of `least` rows or more: the shortest
    // piece has half of `least` (of 256: 320 rows are 128 and 192).  fit_rest: what is
    // left behind whole tiles walks far more than they do (the sinks of a window, that all
    // later rows see), so that its pieces are longer where that takes less.
    void make(std::vector<Range> ranges, int32_t heads, int64_t tile, int64_t unit,
              int64_t least, int64_t slots, double launch = kLaunch, bool fit_rest = false)
    {
        double tiles = 0;
        for (const Range &r : ranges) tiles += (double)ceil_div(r.rows, tile) * heads;
        if (tiles > kMostTiles) {
            parts = INT64_MAX;
            return;
        }
        // the longest first: what is left for the end are short ones
        std::stable_sort(ranges.begin(), ranges.end(),
                         [](const Range &a, const Range &b) { return a.others > b.others; });
        double best = 0;
        int64_t per = best_pieces(ranges, heads, tile, unit, least, slots, launch, &best);
        std::vector<int64_t> most(ranges.size(), per);  // units of a range's pieces
        // A few tiles too many cost a round.  What is left of the ranges behind
        // their whole tiles is then better cut small and run behind the others:
        // 260 tiles of 253 units on 512 places as 512 halves and 4 x 64 pieces
        // instead of 260 x 11 pieces (dK and dV of 2 x 4,050 x 4,050, 16 heads of
        // 128 over 4: 558 us and 22 for their sums instead of 616 and 46).
        std::vector<Range> whole, rest;
        for (const Range &r : ranges) {
            const int64_t n = r.rows / tile * tile;
            if (n) whole.push_back({r.row, n, r.other, r.others, r.tag});
            if (n < r.rows) rest.push_back({r.row + n, r.rows - n, r.other, r.others, r.tag});
        }
        if (!whole.empty() && !rest.empty()) {
            int64_t small = ceil_div(least, unit);
            double t = 0, n = 0;
            if (fit_rest) small = best_rest(rest, heads, unit, small, slots);
            per = best_pieces(whole, heads, tile, unit, least, slots, launch, &t);
            for (const Range &r : rest)
                n += (double)pieces(ceil_div(r.others, unit), small) * heads;
            t += (double)ceil_div((int64_t)n, slots) * (small + kOver + kJoin) +
                 (split(whole, unit, per) ? 0 : launch);
            if (t < kWorth * best) {
                most.assign(whole.size(), per);
                most.resize(whole.size() + rest.size(), small);
                ranges.swap(whole);
                ranges.insert(ranges.end(), rest.begin(), rest.end());
            }
        }
        // The tiles of a sequence, head and piece walk the same rows: they come
        // one behind the other and run side by side, in step, so that a row is
        // fetched once for many of them.  (Shares cut wherever they are equal,
        // which are out of step, took 1.5 times as long; one consecutive range
        // of the items for each XCD instead of every eighth 10% longer: forward,
        // 2 x 4,050 tokens, 32 heads of 128 over 8, 8,100 keys.)
        for (size_t i = 0; i < ranges.size(); ++i) {
            const Range &r = ranges[i];
            const int64_t units = ceil_div(r.others, unit), n = pieces(units, most[i]);
            for (int32_t h = 0; h < heads; ++h) {
                const int64_t part = parts;
                for (int64_t k = 0; k < n; ++k) {
                    const int64_t b = units * k / n * unit;
                    int64_t e = units * (k + 1) / n * unit;
                    if (e > r.others) e = r.others;
                    for (int64_t at = 0; at < r.rows; at += tile) {
                        const int64_t rows = r.rows - at < tile ? r.rows - at : tile;
                        items.push_back({h, (int32_t)(r.row + at), (int32_t)rows,
                                         (int32_t)(r.other + b), (int32_t)(e - b),
                                         n > 1 ? (int32_t)(part + at * n + k * rows) : -1,
                                         (int32_t)k, r.tag});
                    }
                }
                if (n == 1) continue;
                for (int64_t at = 0; at < r.rows; at += tile) {
                    const int64_t rows = r.rows - at < tile ? r.rows - at : tile;
                    merges.push_back({h, (int32_t)(r.row + at), (int32_t)rows,
                                      (int32_t)(part + at * n), (int32_t)rows, (int32_t)n, {}});
                    if (rows > merge_rows) merge_rows = (int32_t)rows;
                }
                parts += r.rows * n;
            }
        }
    }

    bool fits() const
    {
        // (two workgroups to an item, one to four rows of a merge at most)
        return parts <= 0x7FFFFFFF && 2 * (int64_t)items.size() <= kMostGrid &&
               (int64_t)merges.size() * (merge_rows / 4 + 1) <= kMostGrid;
    }
};

}  // namespace f3s
