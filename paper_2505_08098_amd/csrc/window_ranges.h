// The tiles of rows that a window plan hands out, and what each of them walks (host only).
#pragma once

#include <algorithm>
#include <vector>

#include "dense_division.h"

namespace f3s {

constexpr int64_t kWindowTile = 128;  // rows of a tile

// What the items of a range share (its tag).
struct WindowShared {
    int32_t key0, shift;
    WindowKeys keys;
};

// Every tile of rows is a range of its own, since each walks other rows.
struct WindowRanges {
    std::vector<Range> queries, keys;
    std::vector<WindowShared> shared;
};

// The arguments of f3s_window_plan, checked; g query heads to a key head.
inline WindowRanges window_ranges(const int32_t *q_ptr, const int32_t *k_ptr,
                                  const int32_t *q_len, const int32_t *k_len, int32_t n,
                                  int64_t g, const WindowRule &rule)
{
    WindowRanges to;
    for (int32_t b = 0; b < n; ++b) {
        const int64_t q0 = q_ptr[b], k0 = k_ptr[b], q = q_ptr[b + 1] - q0, k = k_ptr[b + 1] - k0;
        const int64_t ql = q_len ? q_len[b] : q, kl = k_len ? k_len[b] : k;
        // position of query token t, as rows are numbered: t + shift
        const int64_t shift = kl - ql - q0;
        auto share = [&](WindowKeys w) {
            to.shared.push_back({(int32_t)k0, (int32_t)shift, w});
            return (int32_t)to.shared.size() - 1;
        };
        for (int64_t r = 0; r < ql * g; r += kWindowTile) {
            const int64_t rows = std::min(kWindowTile, ql * g - r), at = q0 * g + r;
            const WindowKeys w = window_keys(rule, (int32_t)(at / g + shift),
                                             (int32_t)((at + rows - 1) / g + shift), 1);
            to.queries.push_back({at, rows, 0, window_length(w), share(w)});
        }
        // keys: the sinks by themselves (unless the window reaches all of them anyway)
        const int64_t far = rule.window < kl ? std::min<int64_t>(rule.sinks, kl) : 0;
        for (int64_t j = 0; j < kl;) {
            const int64_t rows = std::min(kWindowTile, (j < far ? far : kl) - j);
            // tokens that see the first of them, up to those that see the last
            const int64_t least = std::max<int64_t>(j + ql - kl, 0);
            const int64_t last = j + rows - 1 + rule.window + ql - kl;
            const int64_t most = j < far ? ql : std::min(ql, std::max<int64_t>(last, 0));
            const int64_t tokens = std::max<int64_t>(most - least, 0);
            to.keys.push_back({k0 + j, rows, tokens ? (q0 + least) * g : 0, tokens * g,
                               share({0, 0, 0})});
            j += rows;
        }
        // (rows that are padding walk nothing: their results are zeros)
        if (ql < q) to.queries.push_back({(q0 + ql) * g, (q - ql) * g, 0, 0, share({0, 0, 0})});
        if (kl < k) to.keys.push_back({k0 + kl, k - kl, 0, 0, share({0, 0, 0})});
    }
    return to;
}

}  // namespace f3s
