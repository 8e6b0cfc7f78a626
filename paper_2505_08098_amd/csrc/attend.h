// Attention over the 8-bit cache (f3s_cache_attend): the kernels' arguments,
// shared by their instances (attend_f16.hip, attend_bf16.hip) and the entry
// point (attend.hip).
#pragma once

#include "few_rows.h"

namespace f3s {

// Keys are handed out in units of 64, at least kLeastUnits to a workgroup.
constexpr int kUnit = 64;
constexpr int kLeastUnits = 4;
// Tokens of a sequence's table, or of the prefix.
constexpr int32_t kMostTokens = 1 << 30;

struct AttendArgs {
    FewArgs few;
    const int32_t *table, *lens, *prefix;
    int32_t max_pages, prefix_len;
    int32_t n_seqs, n_new;
    int32_t rows;          // query rows of a sequence and key head: n_new * g
    int32_t row_blocks;    // of 16, of a sequence and key head
    int32_t share;         // workgroups, about, that the own keys of a key head and row
                           // block are divided among
    int32_t own_items;     // workgroups per key head and row block: share + n_seqs
    bool whole;            // or n_seqs: every sequence is one item
    bool direct;           // one workgroup has all keys: no partial results
    // the prefix, all sequences' rows together
    bool prefix_many;       // by the kernel of many rows
    int32_t prefix_blocks;  // row blocks (of 16, or 128) of a key head
    int32_t prefix_splits, prefix_chunk;
    int64_t prefix_part;   // first partial row
    int2 *desc;            // per sequence: its first item and their number
    // what f3s_cache_attend has none of
    int32_t own_rows;      // query rows of a workgroup of the own keys: 16, 128 or 256
    WindowRule rule;
    int32_t splits;        // a window: pieces of every row block's keys
    const int32_t *parents;  // a tree: [n_seqs, n_new]
};

// How the own keys of a batch are divided, from the lengths on the device.
struct OwnItem {
    int32_t seq;     // -1: nothing to do
    int32_t first;   // the sequence's first item
    int32_t items;   // and their number
    int32_t units;   // units of the sequence
    int32_t keys;    // its keys
};

__host__ __device__ inline int32_t units_of(int32_t keys)
{
    return keys / kUnit + (keys % kUnit != 0);
}
// Units to an item where `total` are divided among about `share`.
__host__ __device__ inline int32_t units_per_item(int64_t total, int32_t share)
{
    const int64_t c = (total + share - 1) / share;
    return c < kLeastUnits ? kLeastUnits : (int32_t)c;
}
// Items of a sequence: one also where it has no keys (its rows need a result).
__host__ __device__ inline int32_t items_of(int32_t units, int32_t per_item)
{
    return units <= per_item ? 1 : (units + per_item - 1) / per_item;
}
// First unit of the k-th of n items.
__host__ __device__ inline int32_t item_unit(int32_t units, int32_t k, int32_t n)
{
    return (int32_t)((int64_t)units * k / n);
}

__device__ __forceinline__ int wave_sum(int v)
{
#pragma unroll
    for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
    return v;
}
__device__ __forceinline__ int wave_prefix(int v, int lane)  // inclusive
{
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int u = __shfl_up(v, s);
        if (lane >= s) v += u;
    }
    return v;
}

// Item i of the batch's own keys, divided by `per` units to an item.
__device__ __forceinline__ OwnItem own_item_at(const AttendArgs &a, int i, int per)
{
    const int lane = threadIdx.x & 63;
    const int64_t cap = (int64_t)a.max_pages << a.few.page_shift;
    int before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        const int b = b0 + lane;
        const int keys = b < a.n_seqs ? cache_keys(a.lens[b], cap) : 0;
        const int n = b < a.n_seqs ? items_of(units_of(keys), per) : 0;
        const int upto = wave_prefix(n, lane);
        const uint64_t past = __ballot(before + upto > i);
        if (past) {
            const int at = __builtin_ctzll(past);
            OwnItem o;
            o.seq = b0 + at;
            o.items = __builtin_amdgcn_readlane(n, at);
            o.first = before + __builtin_amdgcn_readlane(upto, at) - o.items;
            o.keys = __builtin_amdgcn_readlane(keys, at);
            o.units = units_of(o.keys);
            return o;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return OwnItem{-1, 0, 0, 0, 0};
}

// Item i (every wave finds it by itself).
__device__ __forceinline__ OwnItem own_item(const AttendArgs &a, int i)
{
    const int lane = threadIdx.x & 63;
    const int64_t cap = (int64_t)a.max_pages << a.few.page_shift;
    if (a.whole) {
        const int32_t keys = cache_keys(a.lens[i], cap);
        return OwnItem{i, i, 1, units_of(keys), keys};
    }
    int total = 0;
    for (int b = lane; b < a.n_seqs; b += 64) total += units_of(cache_keys(a.lens[b], cap));
    return own_item_at(a, i, units_per_item(wave_sum(total), a.share));
}

// Workgroup wg of the prefix: one of its row blocks, key heads and pieces.
__device__ __forceinline__ FewItem prefix_item(const AttendArgs &a, int wg)
{
    FewItem it = {};
    const int rb = wg % a.prefix_blocks, sh = wg / a.prefix_blocks;
    it.head = sh % a.few.n_kv;
    const int split = sh / a.few.n_kv;
    const int64_t all = (int64_t)a.rows * a.n_seqs;
    it.row = (int64_t)rb * kFewRows;
    it.rows = (int)(all - it.row < kFewRows ? all - it.row : kFewRows);
    it.table = a.prefix;
    it.begin = split * a.prefix_chunk;
    it.end = min(a.prefix_len, it.begin + a.prefix_chunk);
    it.table_len = ((a.prefix_len - 1) >> a.few.page_shift) + 1;
    it.causal = false;
    it.part = a.prefix_part + ((int64_t)split * a.few.n_kv + it.head) * all + it.row;
    return it;
}

// Workgroup wg of the own keys; rows = 0 where there is nothing to do.
__device__ __forceinline__ FewItem own_keys_item(const AttendArgs &a, int wg)
{
    FewItem it = {};
    const int rb = wg % a.row_blocks, ih = wg / a.row_blocks;
    it.head = ih % a.few.n_kv;
    const int i = ih / a.few.n_kv;
    const OwnItem o = own_item(a, i);
    if (o.seq < 0) return it;
    const int k = i - o.first;
    if (k == 0 && it.head == 0 && rb == 0 && threadIdx.x == 0 && !a.direct)
        a.desc[o.seq] = int2{o.first, o.items};
    it.row = (int64_t)o.seq * a.rows + rb * kFewRows;
    it.rows = min(kFewRows, a.rows - rb * kFewRows);
    it.table = a.table + (int64_t)o.seq * a.max_pages;
    it.table_len = a.max_pages;
    it.begin = item_unit(o.units, k, o.items) * kUnit;
    it.end = min(o.keys, item_unit(o.units, k + 1, o.items) * kUnit);
    it.causal = a.n_new > 1;
    it.first = rb * kFewRows;
    const int64_t base = cache_position(a.lens[o.seq], a.n_new, 0);
    // (behind the keys that there are, any limit does)
    it.limit = (int)min(base + 1, (int64_t)o.keys);
    it.base = (int)base;
    it.part =
        a.direct ? -1 : ((int64_t)i * a.few.n_kv + it.head) * a.rows + rb * kFewRows;
    return it;
}

// Workgroups of the prefix in the kernel of few rows.
__device__ __forceinline__ int few_prefix(const AttendArgs &a)
{
    return a.prefix_many ? 0 : a.prefix_splits * a.few.n_kv * a.prefix_blocks;
}

template <int D, int kIn>
__global__ __launch_bounds__(64 * kFewWaves, few_waves(D, true)) void k_attend(AttendArgs a)
{
    const int wg = (int)blockIdx.x, n_prefix = few_prefix(a);
    const FewItem it = wg < n_prefix ? prefix_item(a, wg) : own_keys_item(a, wg - n_prefix);
    if (it.rows == 0) return;
    few_rows<D, kIn, true>(a.few, it);
}

// Final results of every row from its partial ones.
template <int D, int kIn, bool kSplit>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a)
{
    constexpr int kPer = kSplit ? 1 : 256 / (D / 4);  // rows of a workgroup
    const int64_t out =
        (int64_t)blockIdx.x * kPer + (kSplit ? 0 : (int)threadIdx.x / (D / 4));
    const int64_t all = (int64_t)a.rows * a.n_seqs;  // of a key head
    if (!kSplit && ((int)threadIdx.x >= kPer * (D / 4) || out >= all * a.few.n_kv)) return;
    const int64_t token = out / a.few.q.n_heads;
    const int h = (int)(out - token * a.few.q.n_heads), kh = h / a.few.q.g;
    const int64_t r = token * a.few.q.g + (h - kh * a.few.q.g);
    const int b = (int)(token / a.n_new);
    const int2 d = a.desc[b];
    const PartRows own = {((int64_t)d.x * a.few.n_kv + kh) * a.rows + (r - (int64_t)b * a.rows),
                          (int64_t)a.few.n_kv * a.rows, d.y};
    const PartRows prefix = {a.prefix_part + kh * all + r, a.few.n_kv * all, a.prefix_splits};
    join_row<D, kIn, kInF16, kSplit>(a.few.part_o, a.few.part_ml, own, prefix, out, a.few.O,
                                     a.few.lse);
}

template <int D, int kIn>
hipError_t launch_attend_prefix_d(const AttendArgs &a, hipStream_t s);

template <int D, int kIn>
void launch_attend_join_d(const AttendArgs &a, hipStream_t s)
{
    if (a.direct) return;
    constexpr int kPer = 256 / (D / 4);
    const int64_t rows = (int64_t)a.rows * a.n_seqs * a.few.n_kv;
    if (rows <= kSplitJoins)
        k_attend_join<D, kIn, true><<<(unsigned)rows, 256, 0, s>>>(a);
    else
        k_attend_join<D, kIn, false><<<(unsigned)((rows + kPer - 1) / kPer), 256, 0, s>>>(a);
}

template <int D, int kIn>
hipError_t launch_attend_d(const AttendArgs &a, hipStream_t s)
{
    int64_t grid = (int64_t)a.own_items * a.few.n_kv * a.row_blocks;
    if (a.prefix_many) {
        const hipError_t e = launch_attend_prefix_d<D, kIn>(a, s);
        if (e != hipSuccess) return e;
    } else {
        grid += (int64_t)a.prefix_splits * a.few.n_kv * a.prefix_blocks;
    }
    k_attend<D, kIn><<<(unsigned)grid, 64 * kFewWaves, 0, s>>>(a);
    launch_attend_join_d<D, kIn>(a, s);
    return hipGetLastError();
}

hipError_t launch_attend_f16(const AttendArgs &a, int d, hipStream_t s);
hipError_t launch_attend_bf16(const AttendArgs &a, int d, hipStream_t s);

}  // namespace f3s
