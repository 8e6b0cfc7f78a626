// f3s_pages_assign: page tables brought from one set of lengths to another, on the device
// (f3s_pages.h).
//
// Per sequence: the pages that it gives back (counted, since an entry may be none) and
// those that it needs; sums of both over the sequences before it, which fix every page's
// place in the pool; then what is given back is appended, and what is needed taken.  A
// wave has one sequence at a time, 64 entries side by side.  Small batches do all of it in
// one workgroup and one launch, since a launch costs more than the work; larger ones in
// four launches (the pool's new end has to stand before any of it is taken).
#include "dense_common.h"
#include "f3s_pages.h"

namespace f3s {

namespace {

constexpr int kFill = 256;      // threads of the launches over sequences
constexpr int kScan = 1024;     // threads of a workgroup by itself
// Sequences, entries of the table and places up to which one workgroup does it all.
constexpr int64_t kAloneSeqs = kScan;
constexpr int64_t kAloneEntries = 1 << 17;
constexpr int64_t kAloneSlots = 1 << 15;
constexpr int32_t kMostSeqs = 1 << 24;

struct PageArgs {
    int32_t *free_pages, *n_free;
    int32_t n_pages;
    int32_t *table;
    int32_t max_pages;
    const int32_t *lens, *new_lens;
    int32_t *got_lens;
    int64_t *slots;
    int32_t n_seqs, n_new, page_shift;
    // workspace: pages given back and needed by every sequence, then by those before it;
    // the pool's size before the call, with what is given back, and what is handed out
    int32_t *back, *need;
    int64_t *sums;
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

// Pages that sequence b gives back: how many there are (a whole wave).
__device__ __forceinline__ int count_back(const PageArgs &a, int b, const Pages &p, int lane)
{
    const int32_t *row = a.table + (int64_t)b * a.max_pages;
    int n = 0;
    for (int e = p.want; e < p.have; e += 64)
        n += __popcll(__ballot(e + lane < p.have && is_page(a, row[min(e + lane, p.have - 1)])));
    return n;
}

// They are appended from place `to` of the pool on, their entries cleared.
__device__ __forceinline__ void give_back(const PageArgs &a, int b, const Pages &p, int64_t to,
                                          int lane)
{
    int32_t *row = a.table + (int64_t)b * a.max_pages;
    for (int e = p.want; e < p.have; e += 64) {
        const bool there = e + lane < p.have;
        const int32_t page = there ? row[e + lane] : -1;
        const uint64_t all = __ballot(is_page(a, page));
        const int64_t at = to + __popcll(all & ((1ull << lane) - 1));
        if (is_page(a, page) && at < a.n_pages) a.free_pages[at] = page;
        if (there) row[e + lane] = -1;
        to += __popcll(all);
    }
}

// Entries have .. want - 1 of sequence b from place `from` of the pool on, as far as it is
// below `end`; then its length and its newest tokens' places.
__device__ __forceinline__ void take(const PageArgs &a, int b, const Pages &p, int64_t from,
                                     int64_t end, int lane)
{
    int32_t *row = a.table + (int64_t)b * a.max_pages;
    for (int e = p.have + lane; e < p.want; e += 64) {
        const int64_t at = from + (e - p.have);
        row[e] = at < end ? a.free_pages[at] : -1;
    }
    const int64_t left = end - from;
    const int32_t kept = min(p.have, p.want);
    const int32_t got_pages =
        kept + (p.want > p.have ? (int32_t)min((int64_t)(p.want - p.have), max(left, (int64_t)0))
                                : 0);
    const int32_t got = (int32_t)min((int64_t)p.length, (int64_t)got_pages << a.page_shift);
    if (lane == 0) a.got_lens[b] = got;
    int64_t *to = a.slots + (int64_t)b * a.n_new;
    for (int t = lane; t < a.n_new; t += 64) {
        const int64_t pos = (int64_t)p.length - a.n_new + t;
        int64_t slot = -1;
        if (pos >= 0 && pos < got) {
            const int32_t e = (int32_t)(pos >> a.page_shift);
            // (entries that are new are read from where they come)
            const int32_t page = e < kept ? row[e] : a.free_pages[from + (e - p.have)];
            if (is_page(a, page))
                slot = ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
        }
        to[t] = slot;
    }
}

// Sums of x and y over the threads before this one, and over all (1024 threads).
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
    for (int w = 0; w < kScan / 64; ++w) {
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
__device__ __forceinline__ Pool pool_of(const PageArgs &a, int64_t back, int64_t need)
{
    const int64_t held = clamped(*a.n_free, a.n_pages);
    const int64_t with = min(held + back, (int64_t)a.n_pages);
    return {held, with, min(need, with)};
}

__global__ __launch_bounds__(kScan) void k_pages_alone(PageArgs a)
{
    __shared__ int64_t s_sum[kScan / 64][2];
    __shared__ int32_t s_back[kScan], s_need[kScan];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = threadIdx.x;
    Pages p = {0, 0, 0};
    if (b < a.n_seqs) p = pages_of(a, b);
    s_back[b] = 0;
    // (a wave counts what each of its 64 sequences gives back)
    for (uint64_t some = __ballot(p.want < p.have); some; some &= some - 1) {
        const int k = __builtin_ctzll(some);
        const Pages its = {__shfl(p.have, k), __shfl(p.want, k), 0};
        const int n = count_back(a, 64 * wave + k, its, lane);
        if (lane == k) s_back[b] = n;
    }
    const int32_t back = s_back[b], need = max(p.want - p.have, 0);
    const Sums sum = sums_before(back, need, s_sum);
    const Pool pool = pool_of(a, sum.all_x, sum.all_y);
    s_back[b] = (int32_t)sum.x;
    s_need[b] = (int32_t)sum.y;
    __syncthreads();  // (everybody has read the pool's size)
    if (threadIdx.x == 0) *a.n_free = (int32_t)(pool.with - pool.given);
    if (sum.all_x) {
        for (int k = wave; k < a.n_seqs; k += kScan / 64) {
            const Pages its = pages_of(a, k);
            if (its.want < its.have) give_back(a, k, its, pool.held + s_back[k], lane);
        }
    }
    __syncthreads();
    for (int k = wave; k < a.n_seqs; k += kScan / 64)
        take(a, k, pages_of(a, k), pool.with - pool.given + s_need[k], pool.with, lane);
}

__global__ __launch_bounds__(kFill) void k_pages_count(PageArgs a)
{
    const int b = (int)blockIdx.x * (kFill / 64) + (int)(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (b >= a.n_seqs) return;
    const Pages p = pages_of(a, b);
    const int n = count_back(a, b, p, lane);
    if (lane) return;
    a.back[b] = n;
    a.need[b] = max(p.want - p.have, 0);
}

__global__ __launch_bounds__(kScan) void k_pages_sum(PageArgs a)
{
    __shared__ int64_t s_sum[kScan / 64][2];
    const int each = (a.n_seqs + kScan - 1) / kScan;
    const int first = min((int)threadIdx.x * each, a.n_seqs), last = min(first + each, a.n_seqs);
    int64_t back = 0, need = 0;
    for (int b = first; b < last; ++b) {
        back += a.back[b];
        need += a.need[b];
    }
    const Sums sum = sums_before(back, need, s_sum);
    const Pool pool = pool_of(a, sum.all_x, sum.all_y);
    // (places in the pool are below 2^31; sums beyond it reach no place)
    back = sum.x, need = sum.y;
    for (int b = first; b < last; ++b) {
        const int32_t x = a.back[b], y = a.need[b];
        a.back[b] = (int32_t)min(back, (int64_t)0x7FFFFFFF);
        a.need[b] = (int32_t)min(need, (int64_t)0x7FFFFFFF);
        back += x;
        need += y;
    }
    __syncthreads();  // (everybody has read the pool's size)
    if (threadIdx.x == 0) {
        a.sums[0] = pool.held;
        a.sums[1] = pool.with;
        a.sums[2] = pool.given;
        *a.n_free = (int32_t)(pool.with - pool.given);
    }
}

__global__ __launch_bounds__(kFill) void k_pages_back(PageArgs a)
{
    const int b = (int)blockIdx.x * (kFill / 64) + (int)(threadIdx.x >> 6);
    if (b >= a.n_seqs) return;
    const Pages p = pages_of(a, b);
    if (p.want < p.have) give_back(a, b, p, a.sums[0] + a.back[b], threadIdx.x & 63);
}

__global__ __launch_bounds__(kFill) void k_pages_take(PageArgs a)
{
    const int b = (int)blockIdx.x * (kFill / 64) + (int)(threadIdx.x >> 6);
    if (b >= a.n_seqs) return;
    const int64_t end = a.sums[1];
    take(a, b, pages_of(a, b), end - a.sums[2] + a.need[b], end, threadIdx.x & 63);
}

bool alone(int32_t n_seqs, int32_t max_pages, int32_t n_new)
{
    return n_seqs <= kAloneSeqs && (int64_t)n_seqs * max_pages <= kAloneEntries &&
           (int64_t)n_seqs * n_new <= kAloneSlots;
}

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && na && nb && x < y + nb && y < x + na;
}

size_t list_bytes(int32_t n_seqs) { return ((size_t)n_seqs * 4 + 15) & ~(size_t)15; }

}  // namespace

}  // namespace f3s

extern "C" {

size_t f3s_pages_assign_workspace_bytes(int32_t n_seqs, int32_t max_pages, int32_t n_new)
{
    if (n_seqs < 1 || max_pages < 0 || n_new < 0 || n_seqs > f3s::kMostSeqs ||
        f3s::alone(n_seqs, max_pages, n_new))
        return 0;
    return 2 * f3s::list_bytes(n_seqs) + 32;
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
    if (n_seqs > f3s::kMostSeqs || (int64_t)max_pages * page_size > 1 << 30)
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
                       nullptr};
    if (!need) {
        f3s::k_pages_alone<<<1, f3s::kScan, 0, stream>>>(a);
        return set_status(f3s::status_of(hipGetLastError()));
    }
    char *w = (char *)workspace;
    a.sums = (int64_t *)w;
    a.back = (int32_t *)(w + 32);
    a.need = (int32_t *)(w + 32 + f3s::list_bytes(n_seqs));
    const unsigned grid = ((unsigned)n_seqs + f3s::kFill / 64 - 1) / (f3s::kFill / 64);
    f3s::k_pages_count<<<grid, f3s::kFill, 0, stream>>>(a);
    f3s::k_pages_sum<<<1, f3s::kScan, 0, stream>>>(a);
    f3s::k_pages_back<<<grid, f3s::kFill, 0, stream>>>(a);
    f3s::k_pages_take<<<grid, f3s::kFill, 0, stream>>>(a);
    return set_status(f3s::status_of(hipGetLastError()));
}

}  // extern "C"
