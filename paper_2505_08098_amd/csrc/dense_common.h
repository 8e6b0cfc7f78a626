// Declarations shared by the dense attention operators: cross attention over
// a ragged batch (cross*.hip) and attention over the 8-bit cache (attend*.hip).
#pragma once

#include "f3s_cache.h"
#include "f3s_cross.h"
#include "kernel_common.h"

namespace f3s {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i2v __attribute__((ext_vector_type(2)));
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
    int32_t pad;
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

namespace f3s {

// Results of an entry point: remembers a failure for f3s_last_error.
f3s_status_t set_status(f3s_status_t s);
f3s_status_t status_of(hipError_t e);
hipError_t limited_malloc(void **p, size_t bytes);

}  // namespace f3s
