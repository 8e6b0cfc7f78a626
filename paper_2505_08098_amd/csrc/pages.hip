// f3s_pages_assign: page tables brought from one set of lengths to another, on the device
// (f3s_pages.h).
//
// Per sequence: the pages that it gives back (counted, since an entry may be none) and
// those that it needs; sums of both over the sequences before it, which fix every page's
// place in the pool; then what is given back is appended, and what is needed taken.  A
// wave has one sequence at a time, 64 entries side by side.  Chains of loads are what this
// takes, not bytes.  Small batches do all of it in one workgroup and one launch, a thread
// to a sequence where it needs a single page and a thread to a token's place; larger ones
// in three launches (the pool's new end has to stand before any of it is taken), of which
// every workgroup sums the counts of all before it by itself, and beyond 16,384 sequences
// in four.  256 sequences that take 5 tokens each, 5.2 us; 4,096 of up to 8,000 tokens of
// which a quarter end and a quarter begin, pages of 16, with 256 places each, 19 us.
#include "dense_common.h"
#include "f3s_pages.h"

namespace f3s {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;  // sequences of a workgroup, in launches over them
// Sequences, entries of the table and places up to which one workgroup does it all.  A call
// in which few sequences change their pages takes half of what the launches do, one in
// which many do several times as long, since a wave goes through those of its 64 sequences
// one behind the other; the former is what a step of generation does.  Us of a call in
// graphs, alone and in launches (one more token each; n more each; half of the batch ends
// or begins; lengths of up to 2,000, pages of 16, n places each):
//      8 sequences, n = 8:    4.7, 10.0;    6.9, 11.1;    7.7, 11.9
//                   n = 256:  5.4, 10.6;    9.5, 11.6;    9.0, 12.4
//     64 sequences, n = 8:    5.7, 11.8;   17.4, 12.2;   29.4, 13.2
//                   n = 64:   7.1, 11.9;   42.9, 12.4;   42.1, 13.4
//                   n = 256: 12.1, 12.7;   47.4, 13.1;   45.6, 14.3
//    256 sequences, n = 1:    8.4, 12.2;    9.4, 13.0;   28.0, 13.7
//                   n = 64:  14.9, 12.2;   50.3, 13.4;   53.1, 13.7
//  1,000 sequences, n = 8:   11.6, 12.4;   28.3, 13.6;   46.3, 13.9
// (64 of up to 32,000 tokens, half turned over: 80.6, 21.3).  Beyond kAloneNew places a
// sequence, which a prompt's part has and a step has not, it loses unless there are few.
constexpr int64_t kAloneSeqs = kThreads;
constexpr int64_t kAloneEntries = 1 << 17;
constexpr int64_t kAloneNew = 32;
constexpr int64_t kAloneSlots = 2048;
constexpr int32_t kMostSeqs = 1 << 24;
constexpr int32_t kMostNew = 1 << 30;  // (a thread's index of a token stays below 2^31)

struct PageArgs {
    int32_t *free_pages, *n_free;
    int32_t n_pages;
    int32_t *table;
    int32_t max_pages;
    const int32_t *lens, *new_lens;
    int32_t *got_lens;
    int64_t *slots;
    int32_t n_seqs, n_new, page_shift;
    // workspace: the pool's size before the call; what every sequence gives back; what
    // each workgroup's sequences give back and need (or, `summed`, those before them, and
    // behind the last all)
    int32_t *held, *back;
    int64_t *blocks;
    bool summed;
};

__device__ __forceinline__ int32_t clamped(int32_t x, int64_t most)
{
    return x < 0 ? 0 : x > most ? (int32_t)most : x;
}

// A sequence's entries before and after.
struct Pages {
    int32_t have, want, length;  // length: the new one
};
__device__ __forceinline__ Pages pages_of(const PageArgs &a, int b)
{
    const int64_t room = (int64_t)a.max_pages << a.page_shift;
    const int32_t round = (1 << a.page_shift) - 1;
    const int32_t was = clamped(a.lens[b], room), is = clamped(a.new_lens[b], room);
    return {(was + round) >> a.page_shift, (is + round) >> a.page_shift, is};
}
__device__ __forceinline__ bool is_page(const PageArgs &a, int32_t page)
{
    return page >= 0 && page < a.n_pages;
}

// Pieces of 64 entries, or places, whose loads are under way together.
constexpr int kAhead = 4;

// Pages that sequence b gives back: how many there are (a whole wave).
__device__ __forceinline__ int count_back(const PageArgs &a, int b, const Pages &p, int lane)
{
    const int32_t *row = a.table + (int64_t)b * a.max_pages;
    int n = 0;
    for (int e = p.want; e < p.have; e += 64 * kAhead) {
        int32_t page[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            page[k] = e + 64 * k + lane < p.have ? row[e + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) n += __popcll(__ballot(is_page(a, page[k])));
    }
    return n;
}

// They are appended from place `to` of the pool on, their entries cleared.
__device__ __forceinline__ void give_back(const PageArgs &a, int b, const Pages &p, int64_t to,
                                          int lane)
{
    int32_t *row = a.table + (int64_t)b * a.max_pages;
    for (int e0 = p.want + lane; e0 - lane < p.have; e0 += 64 * kAhead) {
        int32_t page[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) page[k] = e0 + 64 * k < p.have ? row[e0 + 64 * k] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint64_t all = __ballot(is_page(a, page[k]));
            const int64_t at = to + __popcll(all & ((1ull << lane) - 1));
            if (is_page(a, page[k]) && at < a.n_pages) a.free_pages[at] = page[k];
            if (e0 + 64 * k < p.have) row[e0 + 64 * k] = -1;
            to += __popcll(all);
        }
    }
}

// What a sequence's table holds behind the call: it takes pages from place `from` of the
// pool on, as far as that is below `end`.
struct Taken {
    int32_t kept, have;  // entries that stay, and that there were
    int32_t length, got;
    int64_t from;
};
__device__ __forceinline__ Taken taken_by(const PageArgs &a, const Pages &p, int64_t from,
                                          int64_t end)
{
    const int32_t kept = min(p.have, p.want);
    const int64_t more = min((int64_t)max(p.want - p.have, 0), max(end - from, (int64_t)0));
    const int64_t room = ((int64_t)kept + more) << a.page_shift;
    return {kept, p.have, p.length, (int32_t)min((int64_t)p.length, room), from};
}

// The place of token t of the newest.
__device__ __forceinline__ int64_t slot_of(const PageArgs &a, int b, const Taken &x, int t)
{
    const int64_t pos = (int64_t)x.length - a.n_new + t;
    if (pos < 0 || pos >= x.got) return -1;
    const int32_t e = (int32_t)(pos >> a.page_shift);
    // (entries that are new are read from where they come)
    const int32_t page = e < x.kept ? a.table[(int64_t)b * a.max_pages + e]
                                    : a.free_pages[x.from + (e - x.have)];
    return is_page(a, page)
               ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1))
               : -1;
}

// Entries have .. want - 1 of sequence b (by a whole wave).
__device__ __forceinline__ void take(const PageArgs &a, int b, const Pages &p, int64_t from,
                                     int64_t end, int lane)
{
    int32_t *row = a.table + (int64_t)b * a.max_pages;
    for (int e = p.have + lane; e < p.want; e += 64 * kAhead) {
        int32_t page[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t at = from + (e + 64 * k - p.have);
            page[k] = e + 64 * k < p.want && at < end ? a.free_pages[at] : -1;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (e + 64 * k < p.want) row[e + 64 * k] = page[k];
    }
}

// Sums of x and y over the threads before this one, and over all of the workgroup.
struct Sums {
    int64_t x, y, all_x, all_y;
};
__device__ __forceinline__ Sums sums_before(int64_t x, int64_t y, int64_t (*s)[2])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t ix = x, iy = y;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t ux = __shfl_up((long long)ix, d), uy = __shfl_up((long long)iy, d);
        if (lane >= d) {
            ix += ux;
            iy += uy;
        }
    }
    __syncthreads();
    if (lane == 63) {
        s[wave][0] = ix;
        s[wave][1] = iy;
    }
    __syncthreads();
    Sums r = {ix - x, iy - y, 0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) {
            r.x += s[w][0];
            r.y += s[w][1];
        }
        r.all_x += s[w][0];
        r.all_y += s[w][1];
    }
    return r;
}

// The pool: what it holds, holds with what comes back, and hands out.
struct Pool {
    int64_t held, with, given;
};
__device__ __forceinline__ Pool pool_of(const PageArgs &a, int64_t held, int64_t back,
                                        int64_t need)
{
    const int64_t with = min(held + back, (int64_t)a.n_pages);
    return {held, with, min(need, with)};
}

__global__ __launch_bounds__(kThreads) void k_pages_alone(PageArgs a)
{
    __shared__ int64_t s_sum[kWaves][2];
    __shared__ Taken s_taken[kThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = threadIdx.x;
    const int32_t held = clamped(*a.n_free, a.n_pages);
    Pages p = {0, 0, 0};
    if (b < a.n_seqs) p = pages_of(a, b);
    const uint64_t shrink = __ballot(p.want < p.have);
    int back = 0;
    // (a wave goes through those of its 64 sequences that give any back)
    for (uint64_t some = shrink; some; some &= some - 1) {
        const int k = __builtin_ctzll(some);
        const int n = count_back(a, 64 * wave + k, {__shfl(p.have, k), __shfl(p.want, k), 0}, lane);
        if (lane == k) back = n;
    }
    const Sums sum = sums_before(back, max(p.want - p.have, 0), s_sum);
    const Pool pool = pool_of(a, held, sum.all_x, sum.all_y);
    // (everybody has read the pool's size)
    if (threadIdx.x == 0) *a.n_free = (int32_t)(pool.with - pool.given);
    for (uint64_t some = shrink; some; some &= some - 1) {
        const int k = __builtin_ctzll(some);
        give_back(a, 64 * wave + k, {__shfl(p.have, k), __shfl(p.want, k), 0},
                  pool.held + __shfl((long long)sum.x, k), lane);
    }
    const int64_t from = pool.with - pool.given + sum.y;
    const Taken mine = taken_by(a, p, from, pool.with);
    s_taken[b] = mine;
    if (b < a.n_seqs) a.got_lens[b] = mine.got;
    __syncthreads();  // what was given back is there
    const int need = p.want - p.have;
    if (need == 1)
        a.table[(int64_t)b * a.max_pages + p.have] = from < pool.with ? a.free_pages[from] : -1;
    for (uint64_t some = __ballot(need > 1); some; some &= some - 1) {
        const int k = __builtin_ctzll(some);
        take(a, 64 * wave + k, {__shfl(p.have, k), __shfl(p.want, k), 0},
             __shfl((long long)from, k), pool.with, lane);
    }
    for (int i = threadIdx.x; i < a.n_seqs * a.n_new; i += kThreads) {
        const int its = i / a.n_new;
        a.slots[i] = slot_of(a, its, s_taken[its], i - its * a.n_new);
    }
}

// ---- larger batches: a wave to a sequence -------------------------------------------

__global__ __launch_bounds__(kThreads) void k_pages_count(PageArgs a)
{
    __shared__ int s_count[kWaves][2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int b = (int)blockIdx.x * kWaves + wave;
    int back = 0, need = 0;
    if (b < a.n_seqs) {
        const Pages p = pages_of(a, b);
        back = count_back(a, b, p, lane);
        need = max(p.want - p.have, 0);
        if (lane == 0) a.back[b] = back;
    }
    if (lane == 0) {
        s_count[wave][0] = back;
        s_count[wave][1] = need;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        int64_t all = 0;
        for (int w = 0; w < kWaves; ++w) all += s_count[w][threadIdx.x];
        a.blocks[2 * (int64_t)blockIdx.x + threadIdx.x] = all;
    }
    // (a copy that stays while the last launch writes the new size)
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.held = clamped(*a.n_free, a.n_pages);
}

__device__ __forceinline__ int64_t sum_of(int64_t x)  // (over a wave)
{
#pragma unroll
    for (int s = 1; s < 64; s *= 2) x += __shfl_xor((long long)x, s);
    return x;
}

// The workgroups' counts, one of their own, summed in place.
__global__ __launch_bounds__(kThreads) void k_pages_sum(PageArgs a, int n_blocks)
{
    __shared__ int64_t s_sum[kWaves][2];
    const int each = (n_blocks + kThreads - 1) / kThreads;
    const int first = min((int)threadIdx.x * each, n_blocks), last = min(first + each, n_blocks);
    int64_t back = 0, need = 0;
    for (int k = first; k < last; ++k) {
        back += a.blocks[2 * k];
        need += a.blocks[2 * k + 1];
    }
    const Sums sum = sums_before(back, need, s_sum);
    back = sum.x, need = sum.y;
    for (int k = first; k < last; ++k) {
        const int64_t x = a.blocks[2 * k], y = a.blocks[2 * k + 1];
        a.blocks[2 * k] = back;
        a.blocks[2 * k + 1] = need;
        back += x;
        need += y;
    }
    if (threadIdx.x < 2) a.blocks[2 * n_blocks + threadIdx.x] = threadIdx.x ? sum.all_y : sum.all_x;
}

// What the sequences before this workgroup's give back and need, and all.
__device__ __forceinline__ Sums blocks_before(const PageArgs &a, int64_t (*s)[4])
{
    const int n = (int)gridDim.x, k = (int)blockIdx.x;
    if (a.summed)
        return {a.blocks[2 * k], a.blocks[2 * k + 1], a.blocks[2 * n], a.blocks[2 * n + 1]};
    // (at most as many workgroups as threads)
    const int t = threadIdx.x, wave = t >> 6;
    const int64_t x = t < n ? a.blocks[2 * t] : 0, y = t < n ? a.blocks[2 * t + 1] : 0;
    const int64_t part[4] = {sum_of(t < k ? x : 0), sum_of(t < k ? y : 0), sum_of(x), sum_of(y)};
    if ((t & 63) < 4) s[wave][t & 3] = part[t & 3];
    __syncthreads();
    Sums r = {0, 0, 0, 0};
    for (int w = 0; 64 * w < n; ++w) {
        r.x += s[w][0];
        r.y += s[w][1];
        r.all_x += s[w][2];
        r.all_y += s[w][3];
    }
    return r;
}

__global__ __launch_bounds__(kThreads) void k_pages_back(PageArgs a)
{
    __shared__ int64_t s_sum[kWaves][4];
    const Sums sum = blocks_before(a, s_sum);
    if (sum.all_x == 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int first = (int)blockIdx.x * kWaves, b = first + wave;
    if (b >= a.n_seqs) return;
    const Pages p = pages_of(a, b);
    if (p.want >= p.have) return;
    // (what the workgroup's sequences before b give back)
    const int64_t before = sum_of(lane < wave ? a.back[first + lane] : 0);
    give_back(a, b, p, *a.held + sum.x + before, lane);
}

__global__ __launch_bounds__(kThreads) void k_pages_take(PageArgs a)
{
    __shared__ int64_t s_sum[kWaves][4];
    __shared__ int s_need[kWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int b = (int)blockIdx.x * kWaves + wave;
    Pages p = {0, 0, 0};
    if (b < a.n_seqs) p = pages_of(a, b);
    if (lane == 0) s_need[wave] = max(p.want - p.have, 0);
    const Sums sum = blocks_before(a, s_sum);
    const Pool pool = pool_of(a, *a.held, sum.all_x, sum.all_y);
    __syncthreads();  // (the sequences' needs)
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_free = (int32_t)(pool.with - pool.given);
    if (b >= a.n_seqs) return;
    int64_t from = pool.with - pool.given + sum.y;
    for (int w = 0; w < wave; ++w) from += s_need[w];
    take(a, b, p, from, pool.with, lane);
    const Taken its = taken_by(a, p, from, pool.with);
    if (lane == 0) a.got_lens[b] = its.got;
    int64_t *to = a.slots + (int64_t)b * a.n_new;
    for (int t = lane; t < a.n_new; t += 64 * kAhead) {
        int64_t slot[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            slot[k] = t + 64 * k < a.n_new ? slot_of(a, b, its, t + 64 * k) : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t + 64 * k < a.n_new) to[t + 64 * k] = slot[k];
    }
}

bool alone(int32_t n_seqs, int32_t max_pages, int32_t n_new)
{
    return n_seqs <= kAloneSeqs && (int64_t)n_seqs * max_pages <= kAloneEntries &&
           (n_new <= kAloneNew || (int64_t)n_seqs * n_new <= kAloneSlots);
}

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && na && nb && x < y + nb && y < x + na;
}

size_t list_bytes(int32_t n_seqs) { return ((size_t)n_seqs * 4 + 15) & ~(size_t)15; }

int32_t blocks_of(int32_t n_seqs) { return (n_seqs + kWaves - 1) / kWaves; }

}  // namespace

}  // namespace f3s

extern "C" {

size_t f3s_pages_assign_workspace_bytes(int32_t n_seqs, int32_t max_pages, int32_t n_new)
{
    if (n_seqs < 1 || max_pages < 0 || n_new < 0 || n_seqs > f3s::kMostSeqs ||
        n_new > f3s::kMostNew || f3s::alone(n_seqs, max_pages, n_new))
        return 0;
    return 16 + f3s::list_bytes(n_seqs) + 16 * ((size_t)f3s::blocks_of(n_seqs) + 1);
}

f3s_status_t f3s_pages_assign(int32_t *free_pages, int32_t *n_free, int32_t n_pages,
                              int32_t *table, int32_t max_pages, const int32_t *lens,
                              const int32_t *new_lens, int32_t *got_lens, int64_t *slots,
                              int32_t n_seqs, int32_t n_new, int32_t page_size,
                              void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    using f3s::aligned;
    using f3s::set_status;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)))
        return set_status(F3S_ERR_UNSUPPORTED);
    if (n_pages < 1 || max_pages < 0 || n_seqs < 0 || n_new < 0)
        return set_status(F3S_ERR_INVALID_VALUE);
    if (n_seqs == 0) return F3S_OK;
    if (n_seqs > f3s::kMostSeqs || n_new > f3s::kMostNew ||
        (int64_t)max_pages * page_size > 1 << 30)
        return set_status(F3S_ERR_TOO_LARGE);
    if (!free_pages || !n_free || !lens || !new_lens || !got_lens || (max_pages && !table) ||
        (n_new && !slots) || !aligned(free_pages, 4) || !aligned(n_free, 4) ||
        !aligned(table, 4) || !aligned(lens, 4) || !aligned(new_lens, 4) ||
        !aligned(got_lens, 4) || !aligned(slots, 8))
        return set_status(F3S_ERR_INVALID_VALUE);
    const size_t need = f3s_pages_assign_workspace_bytes(n_seqs, max_pages, n_new);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
        return set_status(F3S_ERR_INVALID_VALUE);
    const size_t lb = (size_t)n_seqs * 4;
    const struct {
        const void *p;
        size_t n;
    } out[] = {{free_pages, (size_t)n_pages * 4}, {n_free, 4}, {table, lb * max_pages},
               {got_lens, lb}, {slots, 2 * lb * n_new}, {workspace, need}},
      in[] = {{lens, lb}, {new_lens, lb}};
    for (const auto &x : out) {
        for (const auto &y : in)
            if (f3s::overlap(x.p, x.n, y.p, y.n)) return set_status(F3S_ERR_INVALID_VALUE);
        for (const auto &y : out)
            if (&x != &y && f3s::overlap(x.p, x.n, y.p, y.n))
                return set_status(F3S_ERR_INVALID_VALUE);
    }
    f3s::PageArgs a = {free_pages, n_free, n_pages, table, max_pages, lens, new_lens, got_lens,
                       slots, n_seqs, n_new, __builtin_ctz(page_size), nullptr, nullptr,
                       nullptr, false};
    if (!need) {
        f3s::k_pages_alone<<<1, f3s::kThreads, 0, stream>>>(a);
        return set_status(f3s::status_of(hipGetLastError()));
    }
    const int32_t blocks = f3s::blocks_of(n_seqs);
    char *w = (char *)workspace;
    a.held = (int32_t *)w;
    a.blocks = (int64_t *)(w + 16);
    a.back = (int32_t *)(w + 16 + 16 * ((size_t)blocks + 1));
    a.summed = blocks > f3s::kThreads;
    f3s::k_pages_count<<<blocks, f3s::kThreads, 0, stream>>>(a);
    if (a.summed) f3s::k_pages_sum<<<1, f3s::kThreads, 0, stream>>>(a, blocks);
    f3s::k_pages_back<<<blocks, f3s::kThreads, 0, stream>>>(a);
    f3s::k_pages_take<<<blocks, f3s::kThreads, 0, stream>>>(a);
    return set_status(f3s::status_of(hipGetLastError()));
}

}  // extern "C"
