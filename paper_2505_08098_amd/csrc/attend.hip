// f3s_cache_attend: checks, the division of the work, workspace.
#include <math.h>
#include <stdlib.h>

#include "attend_many.h"

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
// What a piece of the prefix costs beside its keys (queries, partial results),
// in units of 64 keys.
constexpr int64_t kPieceCost = 3;

constexpr size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

struct Layout {
    int64_t own_rows, prefix_rows;   // partial rows
    size_t ml, desc, bytes;          // byte offsets behind part_o, and the sum
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Everything of the arguments that follows from the sizes; false if a size is
// beyond what the kernels count with.
// prefix_rows: 16 or 128 query rows to a workgroup of the prefix, 0: by the rule.
bool divide(const f3s_cache_t &c, int32_t max_pages, int32_t n_seqs, int32_t n_new,
            int32_t n_heads, int32_t prefix_len, int prefix_rows, AttendArgs *a, Layout *w)
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
    a->row_blocks = (int32_t)ceil_div(rows, f3s::kFewRows);
    const int64_t cap_units = ceil_div(cap, f3s::kUnit);
    a->direct = prefix_len == 0 && cap_units <= kDirectUnits;
    int64_t share = ceil_div(kWorkgroups, (int64_t)c.n_kv_heads * a->row_blocks);
    // (no more than the table has places for)
    const int64_t most = ceil_div(cap_units * n_seqs, f3s::kLeastUnits);
    if (share > most) share = most;
    if (share < 1) share = 1;
    a->share = (int32_t)share;
    a->whole = a->direct || cap_units <= f3s::kLeastUnits || n_seqs > kMostDivided;
    a->own_items = a->whole ? n_seqs : (int32_t)(share + n_seqs);
    if (prefix_rows)
        a->prefix_many = prefix_rows == f3s::kManyRows;
    else
        a->prefix_many = all > kFewPrefixRows &&
                         (double)all * prefix_len * c.n_kv_heads > kManyScores;
    a->prefix_many = a->prefix_many && prefix_len;
    a->prefix_blocks =
        (int32_t)ceil_div(all, a->prefix_many ? f3s::kManyRows : f3s::kFewRows);
    a->prefix_splits = a->prefix_chunk = 0;
    if (prefix_len) {
        const int64_t units = ceil_div(prefix_len, f3s::kUnit);
        const int64_t one = (int64_t)c.n_kv_heads * a->prefix_blocks;  // workgroups, unsplit
        int64_t per;
        if (a->prefix_many) {
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
    if (f3s_status_t st = f3s::check_cache(cache)) return set_status(st);
    if (!sizes_ok(cache, max_pages, n_seqs, n_new, n_heads, prefix_len) || !isfinite(scale))
        return set_status(F3S_ERR_INVALID_VALUE);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return set_status(F3S_ERR_UNSUPPORTED);
    if (n_seqs == 0 || n_new == 0) return F3S_OK;
    if (!Q || !O || !lse || !lens || (max_pages && !table) || (prefix_len && !prefix) ||
        !aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4) || !aligned(lens, 4) ||
        !aligned(table, 4) || !aligned(prefix, 4))
        return set_status(F3S_ERR_INVALID_VALUE);
    AttendArgs a = {};
    Layout w;
    const char *rows = getenv("F3S_PREFIX_ROWS");
    if (!divide(*cache, max_pages, n_seqs, n_new, n_heads, prefix_len,
                rows && *rows ? atoi(rows) : 0, &a, &w))
        return set_status(F3S_ERR_TOO_LARGE);
    if (w.bytes && (!workspace || !aligned(workspace, 256) || workspace_bytes < w.bytes))
        return set_status(F3S_ERR_INVALID_VALUE);
    const int64_t tokens = (int64_t)n_seqs * n_new;
    const size_t qb = (size_t)tokens * n_heads * cache->d * 2, lb = (size_t)tokens * n_heads * 4;
    const size_t cb = (size_t)cache->n_pages * cache->n_kv_heads * cache->page_size;
    const struct {
        const void *p;
        size_t n;
    } in[] = {{Q, qb},
              {cache->k, cb * cache->d},
              {cache->v, cb * cache->d},
              {cache->k_exp, cb},
              {cache->v_exp, cb},
              {table, (size_t)n_seqs * max_pages * 4},
              {lens, (size_t)n_seqs * 4},
              {prefix, ((size_t)prefix_len + cache->page_size - 1) / cache->page_size * 4}};
    // (partial results over lengths or pages that others still read would lead
    // anywhere)
    for (const auto &x : in)
        if (overlaps(O, qb, x.p, x.n) || overlaps(lse, lb, x.p, x.n) ||
            overlaps(workspace, w.bytes, x.p, x.n))
            return set_status(F3S_ERR_INVALID_VALUE);
    if (overlaps(O, qb, lse, lb) || overlaps(O, qb, workspace, w.bytes) ||
        overlaps(lse, lb, workspace, w.bytes))
        return set_status(F3S_ERR_INVALID_VALUE);
    a.table = table;
    a.lens = lens;
    a.prefix = prefix;
    a.few.Q = Q;
    a.few.O = O;
    a.few.lse = lse;
    a.few.q = f3s::query_rows(n_heads, n_heads / cache->n_kv_heads);
    a.few.n_kv = cache->n_kv_heads;
    a.few.sl2 = f3s::scale_log2e(scale);
    a.few.flip = signbit(scale) ? 0x80008000u : 0u;
    a.few.k = (const uint8_t *)cache->k;
    a.few.v = (const uint8_t *)cache->v;
    a.few.k_exp = cache->k_exp;
    a.few.v_exp = cache->v_exp;
    a.few.n_pages = cache->n_pages;
    a.few.page_shift = __builtin_ctz(cache->page_size);
    if (w.bytes) {
        a.few.part_o = (float *)workspace;
        a.few.part_ml = (float *)((char *)workspace + w.ml);
        a.desc = (int2 *)((char *)workspace + w.desc);
    }
    return set_status(f3s::status_of(dtype == F3S_DTYPE_BF16
                                         ? f3s::launch_attend_bf16(a, cache->d, stream)
                                         : f3s::launch_attend_f16(a, cache->d, stream)));
}

}  // extern "C"
