// Declarations shared by the dense attention operators: cross attention over
// a ragged batch (cross*.hip) and attention over the 8-bit cache (attend*.hip).
#pragma once

#include "f3s_cache.h"
#include "f3s_cross.h"
#include "f3s_window.h"
#include "kernel_common.h"

namespace f3s {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i2v __attribute__((ext_vector_type(2)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i2v lds_i2;

// Workgroups of 256 threads that one launch takes (fewer than 2^32 threads).
constexpr int64_t kMostGrid = 0xFFFFFFFF / 256;

// The query rows of one key head: row r (over all tokens) is token r / g,
// query head kh * g + r % g, so the g rows of a token lie one behind the other.
struct QueryRows {
    int32_t n_heads;  // query heads
    int32_t g;        // query heads per key head
    uint32_t mul;     // r / g = (2 r * mul) >> 32 >> shift for every r < 2^31:
    int32_t shift;    // mul = ceil(2^(31 + shift) / g), shift = ceil(log2 g)
};
inline QueryRows query_rows(int32_t n_heads, int32_t g)
{
    int shift = 0;
    while ((1ll << shift) < g) ++shift;
    const uint64_t two = 1ull << (31 + shift);
    return {n_heads, g, (uint32_t)((two + (uint64_t)g - 1) / (uint64_t)g), shift};
}
__host__ __device__ inline uint32_t row_token(const QueryRows &q, uint32_t r)
{
    return (uint32_t)((uint64_t)(2 * r) * q.mul >> 32) >> q.shift;
}
// The row of Q, as [tokens * n_heads, d], of row r (< 2^31).
__device__ __forceinline__ int64_t query_row(const QueryRows &q, int kh, int64_t r)
{
    const uint32_t t = row_token(q, (uint32_t)r);
    return (int64_t)t * (uint32_t)(q.n_heads - q.g) + (uint32_t)r + (uint32_t)(kh * q.g);
}

// |scale| log2 e in 32 bits, the largest number of theirs where it is larger (a
// score of 0 times infinity would be NaN).
inline float scale_log2e(float scale)
{
    const double s = (scale < 0 ? -(double)scale : (double)scale) * 1.4426950408889634;
    return s < 0x1.fffffep127 ? (float)s : 0x1.fffffep127f;
}

// One workgroup's share of a forward or backward pass over a ragged batch.
// Rows are those of the pass's own side (packed query rows of the key head,
// or key rows); others are the rows of the other side that it walks.
struct DenseItem {
    int32_t head;     // key head
    int32_t row;      // first row
    int32_t rows;     // rows
    int32_t other;    // first row of the other side
    int32_t others;   // rows of the other side (0: the results are zeros)
    int32_t part;     // first partial row, -1: the results are final
    int32_t piece;    // which part of a split range
    int32_t tag;      // the range's
};
static_assert(sizeof(DenseItem) == 32, "DenseItem must be 32 bytes");

// Rows of a split range: their partial results are rows part, part + stride,
// ... (count of them), plus the row's index in the range.
struct DenseMerge {
    int32_t head;
    int32_t row;
    int32_t rows;
    int32_t part;
    int32_t stride;
    int32_t count;
    int32_t pad[2];
};
static_assert(sizeof(DenseMerge) == 32, "DenseMerge must be 32 bytes");

// ---- a window of keys --------------------------------------------------------------

// The token at position p sees the key at position j <= p if j is one of the
// sequence's first `sinks` or of the `window` newest ones that p counts among.
struct WindowRule {
    int32_t window, sinks;  // 0 .. 2^30
};
__host__ __device__ inline bool window_sees(const WindowRule &w, int32_t p, int32_t j)
{
    return j <= p && (p - j < w.window || j < w.sinks);
}
// Bits 0 .. n of a word (none for n < 0, all from n = 31 on).
__host__ __device__ inline uint32_t bits_to(int32_t n)
{
    return n < 0 ? 0u : n >= 31 ? ~0u : (2u << n) - 1;
}
// The keys key .. key + 31 that it sees, a bit each.
__host__ __device__ inline uint32_t window_bits(const WindowRule &w, int32_t p, int32_t key)
{
    const int32_t upto = p - key;
    return bits_to(upto) & (~bits_to(upto - w.window) | bits_to(w.sinks - key - 1));
}
// Whether every one of the tokens at first .. last sees every one of the keys key ..
// key + n - 1 (n >= 1); whether none of them sees any.
__host__ __device__ inline bool window_all(const WindowRule &w, int32_t first, int32_t last,
                                           int32_t key, int32_t n)
{
    const int32_t near = key > w.sinks ? key : w.sinks;  // the first that is no sink
    return key + n - 1 <= first && (key + n <= w.sinks || last - near < w.window);
}
__host__ __device__ inline bool window_none(const WindowRule &w, int32_t first, int32_t last,
                                            int32_t key, int32_t n)
{
    return key > last || (first - (key + n - 1) >= w.window && key >= w.sinks);
}

// The keys that some of the tokens at first .. last see, as a list: the `far` sinks
// ahead of the window (keys 0 .. far - 1), filled up to whole units, then the keys
// near .. last.  far is 0 where the window reaches the sinks.
constexpr int32_t kWindowUnit = 64;
struct WindowKeys {
    int32_t far, near, end;
};
__host__ __device__ inline int32_t window_pad(int32_t far)
{
    return (far + kWindowUnit - 1) & ~(kWindowUnit - 1);
}
// `step`: what near is a multiple of (a page's tokens come in 16s).
__host__ __device__ inline WindowKeys window_keys(const WindowRule &w, int32_t first,
                                                  int32_t last, int32_t step)
{
    if (last < 0) return {0, 0, 0};
    if (first < 0) first = 0;
    int32_t near = w.window > first ? 0 : (first - w.window + 1) / step * step;
    if (window_pad(w.sinks) >= near) near = 0;
    return {near ? w.sinks : 0, near, last + 1};
}
__host__ __device__ inline int32_t window_length(const WindowKeys &k)
{
    return window_pad(k.far) + k.end - k.near;
}
// The key at place v of that list, and how many of the list's keys stand from there on
// one behind the other (none where v is one of the places that fill a unit up; a key of
// that number is there all the same).
struct KeyRun {
    int32_t key, left;
};
__host__ __device__ inline KeyRun window_run(const WindowKeys &k, int32_t v)
{
    const int32_t pad = window_pad(k.far);
    return v < pad ? KeyRun{v, k.far - v} : KeyRun{k.near + (v - pad), k.end - k.near - (v - pad)};
}

// A DenseItem of a window plan.  Query rows that walk keys: other and others are places
// of the list `keys`.  Key rows that walk query rows: as in DenseItem.
struct WindowItem : DenseItem {
    int32_t key0;     // the sequence's key 0, as a row of K
    int32_t shift;    // position of a token, less its number (row_token)
    WindowKeys keys;
    int32_t fill[3];
};
static_assert(sizeof(WindowItem) == 64, "WindowItem must be 64 bytes");

// ---- a tree of drafted tokens -------------------------------------------------------

// Tokens of a tree, and the words that hold a bit for each: one of ones ahead of them
// (positions before the tree), one behind, so that 32 bits from any place are two words.
constexpr int kTreeTokens = 256;
constexpr int kTreeWords = kTreeTokens / 32 + 2;

// Where 32 bits from position `pos` on begin, of a tree whose first token stands at `base`:
// bit at % 32 of word at / 32 + 1.  A tile of keys may begin or end behind the last token;
// such places count as the last one, so that both words are the row's.
__host__ __device__ inline int32_t tree_place(int32_t pos, int32_t base)
{
    const int32_t at = pos - base;
    return at < -32 ? -32 : at > kTreeTokens - 1 ? kTreeTokens - 1 : at;
}

// ---- the cache's rules ---------------------------------------------------------

// Biased exponent (the scale is 2^(byte - 127)) of a row whose largest finite
// magnitude is m: the smallest with m <= 448 * 2^(byte - 127).  448 is 1.75 * 2^8.
__host__ __device__ inline uint32_t cache_exponent(float m)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, m);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u);
    return e < 0 ? 0u : (uint32_t)e;
}
// Keys that count of a sequence's length (which the caller may have wrong).
__host__ __device__ inline int32_t cache_keys(int32_t len, int64_t capacity)
{
    return len < 0 ? 0 : len > capacity ? (int32_t)capacity : len;
}
// The row of the cache, in tokens of one head, that a position lies in, or -1
// where it has none (before the start, behind the table, a page that is not one).
__host__ __device__ inline int64_t cache_slot(const int32_t *table, int32_t max_pages,
                                              int32_t n_pages, int page_shift, int64_t pos)
{
    if (pos < 0) return -1;
    const int64_t k = pos >> page_shift;
    if (k >= max_pages) return -1;
    const int32_t page = table[k];
    if (page < 0 || page >= n_pages) return -1;
    return ((int64_t)page << page_shift) + (pos & ((1 << page_shift) - 1));
}
// Position of row t of the n newest of a sequence of (claimed) length len.
__host__ __device__ inline int64_t cache_position(int32_t len, int32_t n, int32_t t)
{
    return (int64_t)(len < 0 ? 0 : len) - n + t;
}

}  // namespace f3s

// A plan of f3s_cross_plan.
struct f3s_cross_plan_s {
    int device = 0;
    int32_t n_heads = 0, n_kv = 0, g = 0, d = 0;
    int64_t q_rows = 0, k_rows = 0;    // rows of Q (tokens) and of K
    void *store = nullptr;             // the lists below, one allocation
    f3s::DenseItem *fwd = nullptr, *dq = nullptr, *dkv = nullptr;
    f3s::DenseMerge *fwd_merge = nullptr, *dq_merge = nullptr, *dkv_merge = nullptr;
    int32_t n_fwd = 0, n_dq = 0, n_dkv = 0;
    int32_t n_fwd_merge = 0, n_dq_merge = 0, n_dkv_merge = 0;
    int32_t fwd_merge_rows = 0, dq_merge_rows = 0, dkv_merge_rows = 0;  // longest
    int64_t fwd_parts = 0, dq_parts = 0, dkv_parts = 0;                 // partial rows
    bool few = false;                  // every item has few rows
};

// A plan of f3s_window_plan, with items of its own kind.
struct f3s_window_plan_s : f3s_cross_plan_s {
    f3s::WindowRule rule = {};
    f3s::WindowItem *window_fwd = nullptr, *window_dq = nullptr, *window_dkv = nullptr;
};

namespace f3s {

// Results of an entry point: remembers a failure for f3s_last_error.
f3s_status_t set_status(f3s_status_t s);
f3s_status_t status_of(hipError_t e);
hipError_t limited_malloc(void **p, size_t bytes);

}  // namespace f3s
