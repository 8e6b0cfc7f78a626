// f3s_cache_attend, f3s_cache_attend_window, f3s_cache_attend_tree: checks, the division
// of the work, workspace.
#include <math.h>
#include <stdlib.h>

#include <algorithm>

#include "attend_masked.h"

namespace f3s {
f3s_status_t check_cache(const f3s_cache_t *c);
}

namespace {

using f3s::AttendArgs;

constexpr int64_t kUnits = 256;  // compute units
// Workgroups that the kernel of few rows aims at, two or three rounds of them, so
// that what is left at the end is short.
constexpr int64_t kWorkgroups = 8 * kUnits;
// The prefix takes the kernel of many rows from more than this many query rows
// of a key head on (below, its tiles would be half empty), and from so many
// scores (rows x keys) that its higher rate pays for a launch of its own.  Calls
// on short own keys, us with 16 rows and with 128:
//   8 key heads of 128, 128 rows: 4.2 M scores 24.4 and 25.4, 8.4 M 36.2 and 30.5
//   8 key heads of  64, 128 rows: 4.2 M scores 18.5 and 19.4, 8.4 M 25.0 and 21.9
//   4 key heads of 256, 256 rows: 4.2 M scores 38.0 and 44.8, 8.4 M 59.4 and 54.7
constexpr int64_t kFewPrefixRows = 64;
constexpr int64_t kManyScores = 6000000;
// Units that a table has room for up to which no sequence is divided (so that one
// launch does).  Calls over 250 to 500 and 445 to 890 own keys, 8 key heads of 128,
// us from one call to the next and from one to the next in a captured graph, whole
// and in pieces:
//    4 sequences: 10.5,  8.5 and 14.6, 10.0;   12.6, 12.2 and 14.5, 10.1
//   16 sequences: 10.5,  8.6 and 14.6, 10.3;   12.6, 12.3 and 14.5, 12.2
//   64 sequences: 14.0, 14.1 and 21.1, 21.0;   19.9, 20.1 and 27.9, 27.9
// (16 of 750 to 1,500 took 21.3 us on the GPU whole and 16.2 in pieces.)  A few
// sequences that fill such a table would gain 2 us from pieces in a graph.
constexpr int64_t kDirectUnits = 14;
// Sequences up to which own keys are divided: every workgroup looks through all
// lengths for its item, which grows with the square of their number.  One new token,
// 8 key heads of 64, in us divided and whole: 8,193 sequences of up to 200 keys
// 3,480 and 270, with one of 131,072 among them 3,477 and 1,016 (1 key head: 597 and
// 45, 616 and 918); 32,768 sequences 50,000 and 1,080.
constexpr int64_t kMostDivided = 8192;
// The same for a tree's own keys by many rows, whose workgroups go through all lengths once
// more for every step of a search (fitted_item).  Trees of 16 tokens, in us divided and
// whole: own keys of 100 to 4,000; of 100 to 1,000, and one sequence of 65,536 among them:
//   8 key heads of 128, 4 heads each:  256 sequences 452, 437;  301, 1,711
//                                    1,024 sequences 2,163, 1,478;  1,548, 2,159
//                                    2,048 sequences 5,089, 2,910;  4,424, 2,841
//   1 key head of 64, 8 heads:         256 sequences 61, 91;  71, 1,240
//                                    1,024 sequences 218, 174;  163, 1,272
//                                    4,096 sequences 1,410, 532;  1,365, 1,432
// (8,192 of 50 to 300, 8 key heads of 64, one of 65,536 among them: 39,460 and 2,953)
constexpr int64_t kMostFitted = 1024;
// What a piece of the prefix costs beside its keys (queries, partial results),
// in units of 64 keys.
constexpr int64_t kPieceCost = 3;

constexpr size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

struct Layout {
    int64_t own_rows, prefix_rows;   // partial rows
    size_t ml, desc, bytes;          // byte offsets behind part_o, and the sum
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Query rows to a workgroup of a masked call's own keys.  The kernel of 16 takes up to 32
// rows of a sequence and key head, and more where all of them are few workgroups; that of
// 256 takes 4,096 and more (d = 96, 128).  Us in graphs over windows of 4,000 keys, 8 key
// heads of 128, with 16, 128 and 256 rows:
//    1 sequence:   64 rows 15.4, 20.6; 192 rows 23.2, 25.4; 256 rows 25.3, 26.3
//   16 sequences:  32 rows 40.6, 43.3;  48 rows 55.2, 47.5;  64 rows 64.6, 49.0
//   64 sequences (of 2,000):  32 rows 69.5, 68.7;  48 rows 95.7, 76.2
// (trees: 32 rows 73.7, 93.1 and 64 rows 137, 108 of 64 sequences)
//    1 sequence:   1,024 rows 40.8, 41.9; 4,096 rows 102.5, 97.8; 8,192 rows 174, 162
//    8 sequences:  1,024 rows 152.5, 156.5; 4,096 rows 581, 570
constexpr int64_t kFewOwnRows = 32;
constexpr int64_t kFewOwnBlocks = 112;
constexpr int64_t kManyOwnRows = 4096;
int own_rows_of(const f3s_cache_t &c, int32_t n_seqs, int64_t rows)
{
    const char *wanted = getenv("F3S_OWN_ROWS");
    const int n = wanted && *wanted ? atoi(wanted) : 0;
    if (n == f3s::kFewRows || n == f3s::kManyRows ||
        (n == 2 * f3s::kManyRows && f3s::own_wide(c.d)))
        return n;
    if (rows <= kFewOwnRows ||
        (double)n_seqs * c.n_kv_heads * (double)ceil_div(rows, f3s::kFewRows) <= kFewOwnBlocks)
        return f3s::kFewRows;
    return f3s::own_wide(c.d) && rows >= kManyOwnRows ? 2 * f3s::kManyRows : f3s::kManyRows;
}
// Workgroups that run at once.
int64_t own_slots(int32_t d, int own_rows)
{
    return kUnits * f3s::own_groups(d, own_rows / 32);
}
// What one of its workgroups costs beside its keys, in units of 64 keys, and what a byte of
// partial results does (2.7 us a unit of 128 values; 5 TB/s).
constexpr int64_t kOwnCost = 4;
constexpr double kUnitTime = 2.7e-6, kPartRate = 5e12;
// A prefix in the launch of a tree's own keys fills up what these leave idle: in pieces of
// this many units, but no more of them than make two rounds of workgroups (a long prefix
// has work enough, and every piece of a row is joined).  Us a call in graphs, trees of 63
// tokens, 32 heads of 128 over 8, in pieces of 16 units; by two rounds; in a launch apart:
//   16 trees, own keys of 500 to 8,192 behind 2,001:   155, 153, 173;  behind 16,000: 470, 414, 411
//   4 behind 4,001: 77, 76, 82;  32 of 500 to 4,000 behind 4,001: 309, 288, 297
//   16 of 100 to 500 behind 8,001: 208, 193, 186;  64 of 100 to 3,000 behind 6,001: 718, 622, 632
//   64 of 32 tokens, d = 64, behind 8,001: 255, 239, 242;  2 of 200 behind 60,000: 818, 725, 733
// (8 units and two rounds: 162 for the first, 71 instead of 78 for 8 trees, 16 heads of 96
// over 2, behind 4,001; of three rounds, none but 16 trees of 256 tokens and 16 heads over 1
// gains: 520 for 551)
constexpr int64_t kBesideUnits = 16;
constexpr int64_t kBesideRounds = 2;
// Units of a piece of a window, at least, where the workgroups fill the GPU without it.
constexpr int64_t kWorthUnits = 16;

// Everything of the arguments that follows from the sizes; false if a size is
// beyond what the kernels count with.
// prefix_rows: 16 or 128 query rows to a workgroup of the prefix, 0: by the rule; own_rows:
// those of one of the own keys.
bool divide(const f3s_cache_t &c, int32_t max_pages, int32_t n_seqs, int32_t n_new,
            int32_t n_heads, int32_t prefix_len, int prefix_rows, AttendArgs *a, Layout *w,
            int own_rows = f3s::kFewRows)
{
    // (a key's number and a piece's length add up to less than 2^31)
    if ((double)n_new * n_heads * n_seqs > 0x7FFFFFFF || prefix_len > f3s::kMostTokens ||
        (double)max_pages * c.page_size > f3s::kMostTokens ||
        (double)max_pages * c.page_size / f3s::kUnit * n_seqs + n_seqs > 1e9)
        return false;
    const int64_t g = n_heads / c.n_kv_heads;
    const int64_t rows = n_new * g, all = rows * n_seqs;
    const int64_t cap = (int64_t)max_pages * c.page_size;
    a->n_seqs = n_seqs;
    a->n_new = n_new;
    a->max_pages = max_pages;
    a->prefix_len = prefix_len;
    a->rows = (int32_t)rows;
    a->own_rows = own_rows;
    a->row_blocks = (int32_t)ceil_div(rows, own_rows);
    const int64_t cap_units = ceil_div(cap, f3s::kUnit);
    a->direct = prefix_len == 0 && cap_units <= kDirectUnits;
    int64_t share = ceil_div(kWorkgroups, (int64_t)c.n_kv_heads * a->row_blocks);
    // (no more than the table has places for)
    const int64_t most = ceil_div(cap_units * n_seqs, f3s::kLeastUnits);
    if (share > most) share = most;
    if (share < 1) share = 1;
    a->share = (int32_t)share;
    a->whole = a->direct || cap_units <= f3s::kLeastUnits ||
               n_seqs > (own_rows > f3s::kFewRows ? kMostFitted : kMostDivided);
    a->own_items = a->whole ? n_seqs : (int32_t)(share + n_seqs);
    if (own_rows > f3s::kFewRows && !a->whole) {
        // one round of workgroups, or half as many again as sequences
        const int64_t fit = own_slots(c.d, own_rows) / ((int64_t)c.n_kv_heads * a->row_blocks);
        a->own_items = (int32_t)std::max<int64_t>(fit, n_seqs + n_seqs / 2);
    }
    if (prefix_rows)
        a->prefix_many = prefix_rows == f3s::kManyRows;
    else
        a->prefix_many = all > kFewPrefixRows &&
                         (double)all * prefix_len * c.n_kv_heads > kManyScores;
    a->prefix_many = a->prefix_many && prefix_len;
    // (a tree's many rows take the prefix in the launch of the own keys)
    const bool beside = own_rows > f3s::kFewRows && a->prefix_many;
    a->prefix_blocks = (int32_t)ceil_div(all, beside           ? own_rows
                                              : a->prefix_many ? f3s::kManyRows
                                                               : f3s::kFewRows);
    a->prefix_splits = a->prefix_chunk = 0;
    if (prefix_len) {
        const int64_t units = ceil_div(prefix_len, f3s::kUnit);
        const int64_t one = (int64_t)c.n_kv_heads * a->prefix_blocks;  // workgroups, unsplit
        int64_t per;
        if (beside) {
            const int64_t fill = kBesideRounds * own_slots(c.d, own_rows) / one;
            per = ceil_div(units, std::min(ceil_div(units, kBesideUnits),
                                           std::max<int64_t>(fill, 1)));
        } else if (a->prefix_many) {
            // pieces that fill their rounds, at most kMostChunk keys each
            const int64_t slots = kUnits * f3s::many_waves(c.d);
            double best = INFINITY;
            per = units;
            for (int64_t n = 1; n <= units; ++n) {
                const int64_t p = ceil_div(units, n);
                if (n > 1 && p < f3s::kLeastUnits) break;
                if (p * f3s::kUnit > f3s::kMostChunk) continue;
                const double t = (double)ceil_div(one * ceil_div(units, p), slots) *
                                 (double)(p + kPieceCost);
                if (t < best) {
                    best = t;
                    per = p;
                }
                if (one * n > 4 * slots) break;
            }
        } else {
            per = f3s::units_per_item(units, (int32_t)ceil_div(kWorkgroups, one));
        }
        a->prefix_chunk = (int32_t)(per * f3s::kUnit);
        a->prefix_splits = (int32_t)ceil_div(units, per);
    }
    const int64_t items = (int64_t)a->own_items * c.n_kv_heads;
    w->own_rows = a->direct ? 0 : items * rows;
    w->prefix_rows = (int64_t)a->prefix_splits * c.n_kv_heads * all;
    a->prefix_part = w->own_rows;
    const int64_t n = w->own_rows + w->prefix_rows;
    // (a join has four rows or more to a workgroup where there are many)
    if (items * a->row_blocks + (int64_t)a->prefix_splits * c.n_kv_heads * a->prefix_blocks >
            f3s::kMostGrid ||
        all * c.n_kv_heads / 4 >= f3s::kMostGrid)
        return false;
    w->ml = round256((size_t)n * c.d * 4);
    w->desc = w->ml + round256((size_t)n * 8);
    w->bytes = a->direct ? 0 : w->desc + round256((size_t)n_seqs * 8);
    return true;
}

// The same for a window: the pieces of a row block's keys follow from the longest list of
// keys that one can have, and every sequence has as many.
bool divide_window(const f3s_cache_t &c, int32_t max_pages, int32_t n_seqs, int32_t n_new,
                   int32_t n_heads, const f3s::WindowRule &rule, AttendArgs *a, Layout *w)
{
    if ((double)n_new * n_heads * n_seqs > 0x7FFFFFFF ||
        (double)max_pages * c.page_size > f3s::kMostTokens)
        return false;
    const int64_t g = n_heads / c.n_kv_heads, rows = n_new * g;
    a->n_seqs = n_seqs;
    a->n_new = n_new;
    a->max_pages = max_pages;
    a->rows = (int32_t)rows;
    a->rule = rule;
    a->own_rows = own_rows_of(c, n_seqs, rows);
    const int64_t tile = a->own_rows;
    a->row_blocks = (int32_t)ceil_div(rows, tile);
    const int64_t tokens = std::min<int64_t>(n_new, tile / g + 2);
    const int64_t longest =
        std::min<int64_t>((int64_t)max_pages * c.page_size,
                          (int64_t)f3s::window_pad(rule.sinks) + rule.window + tokens + 15);
    const int64_t units = ceil_div(longest, f3s::kUnit);
    const int64_t one = (int64_t)n_seqs * c.n_kv_heads * a->row_blocks;  // workgroups, unsplit
    int64_t splits = 1;
    if (a->own_rows > f3s::kFewRows) {
        // whole rounds of workgroups, and what the pieces' results cost
        const int64_t slots = own_slots(c.d, a->own_rows);
        double best = INFINITY;
        for (int64_t n = 1;
             n == 1 || (n <= units / f3s::kLeastUnits && one * n <= 4 * slots); ++n) {
            const double join = n == 1 ? 0.0
                                       : 2 + (double)one * n * tile * (c.d + 2) * 8 /
                                                 kPartRate / (kUnitTime * c.d / 128);
            const double t =
                (double)ceil_div(one * n, slots) * (double)(ceil_div(units, n) + kOwnCost) + join;
            if (t < best) {
                best = t;
                splits = n;
            }
        }
    } else if (units > kDirectUnits) {
        // As many workgroups as run at once.  One token over windows of 1,024, 4,096 and
        // 16,384 keys, 8 key heads of 128, us by number of pieces:
        //    8 sequences, 16 units: 15.7 whole, 13.3 (2), 10.8 (4)
        //   32 sequences, 16 units: 18.3 whole, 20.2 (2), 23.5 (4)
        //    8 sequences, 64 units: 51.1 whole, 21.3 (4), 20.3 (12), 22.3 (16)
        //   64 sequences, 64 units: 104 whole, 117 (2), 107 (3), 113 (4)
        //   16 sequences, 256 units: 222 whole, 105 (4), 103 (6), 110 (16)
        const int64_t aim = kUnits * f3s::few_waves(c.d, true);
        const int64_t least = one < kUnits ? (int64_t)f3s::kLeastUnits : kWorthUnits;
        splits = std::max<int64_t>(std::min(aim / one, units / least), 1);
    }
    a->splits = (int32_t)splits;
    a->direct = splits == 1;
    w->own_rows = a->direct ? 0 : (int64_t)n_seqs * splits * c.n_kv_heads * rows;
    w->prefix_rows = 0;
    if ((double)one * (double)splits > (double)f3s::kMostGrid ||
        rows * n_seqs * c.n_kv_heads / 4 >= f3s::kMostGrid)
        return false;
    w->ml = round256((size_t)w->own_rows * c.d * 4);
    w->desc = w->ml + round256((size_t)w->own_rows * 8);
    w->bytes = a->direct ? 0 : w->desc + round256((size_t)n_seqs * 8);
    return true;
}

// And for a tree.
bool divide_tree(const f3s_cache_t &c, int32_t max_pages, int32_t n_seqs, int32_t n_new,
                 int32_t n_heads, int32_t prefix_len, int prefix_rows, AttendArgs *a, Layout *w)
{
    const int64_t rows = (int64_t)n_new * (n_heads / c.n_kv_heads);
    return divide(c, max_pages, n_seqs, n_new, n_heads, prefix_len, prefix_rows, a, w,
                  own_rows_of(c, n_seqs, rows));
}

bool sizes_ok(const f3s_cache_t *c, int32_t max_pages, int32_t n_seqs, int32_t n_new,
              int32_t n_heads, int32_t prefix_len)
{
    return c && c->n_kv_heads >= 1 && c->page_size >= 1 && c->d >= 1 && max_pages >= 0 &&
           n_seqs >= 0 && n_new >= 0 && n_heads >= 1 && n_heads % c->n_kv_heads == 0 &&
           prefix_len >= 0;
}

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na && nb && x < y + nb && y < x + na;
}

// What a call passes, as the entry points have it.
struct Call {
    const f3s_cache_t *cache;
    const void *Q;
    f3s_dtype_t dtype;
    void *O;
    float *lse;
    const int32_t *table;
    int32_t max_pages;
    const int32_t *lens;
    int32_t n_seqs, n_new, n_heads;
    const int32_t *prefix;
    int32_t prefix_len;
    const int32_t *parents;  // a tree's, or NULL
    float scale;
    void *workspace;
    size_t workspace_bytes;
};

// The checks ahead of the division.
f3s_status_t check_call(const Call &x)
{
    if (f3s_status_t st = f3s::check_cache(x.cache)) return st;
    if (!sizes_ok(x.cache, x.max_pages, x.n_seqs, x.n_new, x.n_heads, x.prefix_len) ||
        !isfinite(x.scale))
        return F3S_ERR_INVALID_VALUE;
    if (x.dtype != F3S_DTYPE_F16 && x.dtype != F3S_DTYPE_BF16) return F3S_ERR_UNSUPPORTED;
    if (x.n_seqs == 0 || x.n_new == 0) return F3S_OK;
    if (!x.Q || !x.O || !x.lse || !x.lens || (x.max_pages && !x.table) ||
        (x.prefix_len && !x.prefix) || !aligned(x.Q, 16) || !aligned(x.O, 16) ||
        !aligned(x.lse, 4) || !aligned(x.lens, 4) || !aligned(x.table, 4) ||
        !aligned(x.prefix, 4) || !aligned(x.parents, 4))
        return F3S_ERR_INVALID_VALUE;
    return F3S_OK;
}

// Those behind it, and the arguments that are left.
f3s_status_t finish_call(const Call &x, const Layout &w, AttendArgs *a)
{
    if (w.bytes &&
        (!x.workspace || !aligned(x.workspace, 256) || x.workspace_bytes < w.bytes))
        return F3S_ERR_INVALID_VALUE;
    const f3s_cache_t *cache = x.cache;
    const int64_t tokens = (int64_t)x.n_seqs * x.n_new;
    const size_t qb = (size_t)tokens * x.n_heads * cache->d * 2;
    const size_t lb = (size_t)tokens * x.n_heads * 4;
    const size_t cb = (size_t)cache->n_pages * cache->n_kv_heads * cache->page_size;
    const struct {
        const void *p;
        size_t n;
    } in[] = {{x.Q, qb},
              {cache->k, cb * cache->d},
              {cache->v, cb * cache->d},
              {cache->k_exp, cb},
              {cache->v_exp, cb},
              {x.table, (size_t)x.n_seqs * x.max_pages * 4},
              {x.lens, (size_t)x.n_seqs * 4},
              {x.prefix, ((size_t)x.prefix_len + cache->page_size - 1) / cache->page_size * 4},
              {x.parents, x.parents ? (size_t)tokens * 4 : 0}};
    // (partial results over lengths or pages that others still read would lead
    // anywhere)
    for (const auto &y : in)
        if (overlaps(x.O, qb, y.p, y.n) || overlaps(x.lse, lb, y.p, y.n) ||
            overlaps(x.workspace, w.bytes, y.p, y.n))
            return F3S_ERR_INVALID_VALUE;
    if (overlaps(x.O, qb, x.lse, lb) || overlaps(x.O, qb, x.workspace, w.bytes) ||
        overlaps(x.lse, lb, x.workspace, w.bytes))
        return F3S_ERR_INVALID_VALUE;
    a->table = x.table;
    a->lens = x.lens;
    a->prefix = x.prefix;
    a->parents = x.parents;
    a->few.Q = x.Q;
    a->few.O = x.O;
    a->few.lse = x.lse;
    a->few.q = f3s::query_rows(x.n_heads, x.n_heads / cache->n_kv_heads);
    a->few.n_kv = cache->n_kv_heads;
    a->few.sl2 = f3s::scale_log2e(x.scale);
    a->few.flip = signbit(x.scale) ? 0x80008000u : 0u;
    a->few.k = (const uint8_t *)cache->k;
    a->few.v = (const uint8_t *)cache->v;
    a->few.k_exp = cache->k_exp;
    a->few.v_exp = cache->v_exp;
    a->few.n_pages = cache->n_pages;
    a->few.page_shift = __builtin_ctz(cache->page_size);
    if (w.bytes) {
        a->few.part_o = (float *)x.workspace;
        a->few.part_ml = (float *)((char *)x.workspace + w.ml);
        a->desc = (int2 *)((char *)x.workspace + w.desc);
    }
    return F3S_OK;
}

// F3S_PREFIX_ROWS, or 0.
int prefix_rows_wanted()
{
    const char *rows = getenv("F3S_PREFIX_ROWS");
    return rows && *rows ? atoi(rows) : 0;
}

// A window's numbers (a larger one is this one: positions are below 2^31).
f3s::WindowRule window_rule(int32_t window, int32_t sinks)
{
    return {std::min(window, f3s::kMostTokens), std::min(sinks, f3s::kMostTokens)};
}

}  // namespace

extern "C" {

size_t f3s_cache_attend_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                        int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                        int32_t prefix_len)
{
    if (!sizes_ok(cache, max_pages, n_seqs, n_new, n_heads, prefix_len) || n_seqs == 0 ||
        n_new == 0)
        return 0;
    // (enough for both kernels of the prefix)
    size_t most = 0;
    for (int rows : {f3s::kFewRows, f3s::kManyRows}) {
        AttendArgs a = {};
        Layout w;
        if (!divide(*cache, max_pages, n_seqs, n_new, n_heads, prefix_len, rows, &a, &w))
            return 0;
        if (w.bytes > most) most = w.bytes;
    }
    return most;
}

f3s_status_t f3s_cache_attend(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                              void *O, float *lse, const int32_t *table, int32_t max_pages,
                              const int32_t *lens, int32_t n_seqs, int32_t n_new,
                              int32_t n_heads, const int32_t *prefix, int32_t prefix_len,
                              float scale, void *workspace, size_t workspace_bytes,
                              hipStream_t stream)
{
    using f3s::set_status;
    const Call x = {cache, Q, dtype, O, lse, table, max_pages, lens, n_seqs, n_new, n_heads,
                    prefix, prefix_len, nullptr, scale, workspace, workspace_bytes};
    if (f3s_status_t st = check_call(x)) return set_status(st);
    if (n_seqs == 0 || n_new == 0) return F3S_OK;
    AttendArgs a = {};
    Layout w;
    if (!divide(*cache, max_pages, n_seqs, n_new, n_heads, prefix_len, prefix_rows_wanted(), &a,
                &w))
        return set_status(F3S_ERR_TOO_LARGE);
    if (f3s_status_t st = finish_call(x, w, &a)) return set_status(st);
    return set_status(f3s::status_of(dtype == F3S_DTYPE_BF16
                                         ? f3s::launch_attend_bf16(a, cache->d, stream)
                                         : f3s::launch_attend_f16(a, cache->d, stream)));
}

size_t f3s_cache_attend_window_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                               int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                               int32_t window, int32_t sinks)
{
    if (!sizes_ok(cache, max_pages, n_seqs, n_new, n_heads, 0) || n_seqs == 0 || n_new == 0 ||
        window < 0 || sinks < 0)
        return 0;
    AttendArgs a = {};
    Layout w;
    return divide_window(*cache, max_pages, n_seqs, n_new, n_heads, window_rule(window, sinks),
                         &a, &w)
               ? w.bytes
               : 0;
}

f3s_status_t f3s_cache_attend_window(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                                     void *O, float *lse, const int32_t *table,
                                     int32_t max_pages, const int32_t *lens, int32_t n_seqs,
                                     int32_t n_new, int32_t n_heads, int32_t window,
                                     int32_t sinks, float scale, void *workspace,
                                     size_t workspace_bytes, hipStream_t stream)
{
    using f3s::set_status;
    const Call x = {cache, Q, dtype, O, lse, table, max_pages, lens, n_seqs, n_new, n_heads,
                    nullptr, 0, nullptr, scale, workspace, workspace_bytes};
    if (f3s_status_t st = check_call(x)) return set_status(st);
    if (window < 0 || sinks < 0) return set_status(F3S_ERR_INVALID_VALUE);
    if (n_seqs == 0 || n_new == 0) return F3S_OK;
    AttendArgs a = {};
    Layout w;
    if (!divide_window(*cache, max_pages, n_seqs, n_new, n_heads, window_rule(window, sinks), &a,
                       &w))
        return set_status(F3S_ERR_TOO_LARGE);
    if (f3s_status_t st = finish_call(x, w, &a)) return set_status(st);
    return set_status(
        f3s::status_of(dtype == F3S_DTYPE_BF16
                           ? f3s::launch_attend_window_bf16(a, cache->d, stream)
                           : f3s::launch_attend_window_f16(a, cache->d, stream)));
}

size_t f3s_cache_attend_tree_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                             int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                             int32_t prefix_len)
{
    if (!sizes_ok(cache, max_pages, n_seqs, n_new, n_heads, prefix_len) || n_seqs == 0 ||
        n_new == 0 || n_new > f3s::kTreeTokens)
        return 0;
    // (enough for both kernels of the prefix)
    size_t most = 0;
    for (int rows : {f3s::kFewRows, f3s::kManyRows}) {
        AttendArgs a = {};
        Layout w;
        if (!divide_tree(*cache, max_pages, n_seqs, n_new, n_heads, prefix_len, rows, &a, &w))
            return 0;
        most = std::max(most, w.bytes);
    }
    return most;
}

f3s_status_t f3s_cache_attend_tree(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                                   void *O, float *lse, const int32_t *table, int32_t max_pages,
                                   const int32_t *lens, int32_t n_seqs, int32_t n_new,
                                   int32_t n_heads, const int32_t *parents,
                                   const int32_t *prefix, int32_t prefix_len, float scale,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    using f3s::set_status;
    const Call x = {cache, Q, dtype, O, lse, table, max_pages, lens, n_seqs, n_new, n_heads,
                    prefix, prefix_len, parents, scale, workspace, workspace_bytes};
    if (f3s_status_t st = check_call(x)) return set_status(st);
    if (n_new > f3s::kTreeTokens) return set_status(F3S_ERR_UNSUPPORTED);
    if (n_seqs == 0 || n_new == 0) return F3S_OK;
    if (!parents) return set_status(F3S_ERR_INVALID_VALUE);
    AttendArgs a = {};
    Layout w;
    if (!divide_tree(*cache, max_pages, n_seqs, n_new, n_heads, prefix_len, prefix_rows_wanted(),
                     &a, &w))
        return set_status(F3S_ERR_TOO_LARGE);
    if (f3s_status_t st = finish_call(x, w, &a)) return set_status(st);
    return set_status(
        f3s::status_of(dtype == F3S_DTYPE_BF16
                           ? f3s::launch_attend_tree_bf16(a, cache->d, stream)
                           : f3s::launch_attend_tree_f16(a, cache->d, stream)));
}

}  // extern "C"
