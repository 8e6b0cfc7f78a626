// Writing rows of keys and values into the paged 8-bit cache, reading them back, and
// moving those of accepted tokens (f3s_cache_write, f3s_cache_read, f3s_cache_keep; the
// format is in f3s_cache.h).
//
// Writing and reading are bound by the bytes they move.  The lanes of one row hold 8 of its
// elements each, so that a row's 16-bit side is one 16-byte access per lane
// and its codes one 8-byte access; the largest magnitude goes over those
// lanes.  Each group of lanes takes the K and the V row of its token and key
// head: their place in the cache is looked up once, and both are in flight
// together.  4 x 8,192 tokens, 8 key heads of 128 in bf16: 43 us written, 31 read
// back, 5 TB/s.
#include "dense_common.h"

namespace f3s {

namespace {

constexpr int kThreads = 256;

// Lanes of a row: d / 8, up to the next power of two.
constexpr int lanes_of(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32; }

struct RowArgs {
    f3s_cache_t c;
    const int32_t *table;
    const int32_t *lens;
    int32_t max_pages;
    int32_t page_shift;
    int32_t n_new;
    uint32_t rows;  // sequences * n_new * key heads
};

// The cache row (in rows of d) of row r = (b * n_new + t) * n_kv_heads + kh, or -1.
__device__ __forceinline__ int64_t row_place(const RowArgs &a, uint32_t r)
{
    const uint32_t bt = r / (uint32_t)a.c.n_kv_heads, kh = r - bt * (uint32_t)a.c.n_kv_heads;
    const uint32_t b = bt / (uint32_t)a.n_new, t = bt - b * (uint32_t)a.n_new;
    const int64_t slot =
        cache_slot(a.table + (int64_t)b * a.max_pages, a.max_pages, a.c.n_pages, a.page_shift,
                   cache_position(a.lens[b], a.n_new, (int32_t)t));
    if (slot < 0) return -1;
    const int64_t page = slot >> a.page_shift;
    return ((page * a.c.n_kv_heads + kh) << a.page_shift) +
           (slot & ((1 << a.page_shift) - 1));
}

__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

template <int L>
__device__ __forceinline__ float max_over(float v)
{
#pragma unroll
    for (int s = 1; s < L; s *= 2) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void k_cache_write(RowArgs a, const T *K, const T *V)
{
    constexpr int L = lanes_of(D);
    typedef T t8 __attribute__((ext_vector_type(8)));
    const uint32_t r = blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const int c = threadIdx.x % L;
    if (r >= a.rows) return;  // (whole groups of L lanes)
    const int64_t place = row_place(a, r);
    if (place < 0) return;
    const bool there = L * 8 == D || c * 8 < D;
    const int64_t from = (int64_t)r * D + c * 8;
    t8 x[2] = {};
    if (there) {
        x[0] = *reinterpret_cast<const t8 *>(K + from);
        x[1] = *reinterpret_cast<const t8 *>(V + from);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float v[8], m = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[k] = widen(x[w][k]);
            const float y = fabsf(v[k]);
            m = fmaxf(m, y < INFINITY ? y : 0.f);
        }
        const uint32_t e = cache_exponent(max_over<L>(m));
        u2 codes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = __builtin_ldexpf(v[4 * k + j], 127 - (int)e);
            int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            codes[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
        }
        uint8_t *to = reinterpret_cast<uint8_t *>(w ? a.c.v : a.c.k);
        if (there) *reinterpret_cast<u2 *>(to + place * D + c * 8) = codes;
        if (c == 0) (w ? a.c.v_exp : a.c.k_exp)[place] = (uint8_t)e;
    }
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void k_cache_read(RowArgs a, T *K, T *V)
{
    constexpr int L = lanes_of(D);
    typedef T t8 __attribute__((ext_vector_type(8)));
    const uint32_t r = blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const int c = threadIdx.x % L;
    if (r >= a.rows || (L * 8 != D && c * 8 >= D)) return;
    const int64_t place = row_place(a, r);
    const int64_t to = (int64_t)r * D + c * 8;
    u2 codes[2] = {u2{0, 0}, u2{0, 0}};
    int e[2] = {0, 0};
    if (place >= 0) {
        const uint8_t *k = reinterpret_cast<const uint8_t *>(a.c.k) + place * D + c * 8;
        const uint8_t *v = reinterpret_cast<const uint8_t *>(a.c.v) + place * D + c * 8;
        codes[0] = *reinterpret_cast<const u2 *>(k);
        codes[1] = *reinterpret_cast<const u2 *>(v);
        e[0] = a.c.k_exp[place];
        e[1] = a.c.v_exp[place];
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        T *out = w ? V : K;
        if (!out) continue;
        t8 x;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w][k], false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w][k], true);
            const float y[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[4 * k + j] = (T)__builtin_ldexpf(y[j], e[w] - 127);
        }
        *reinterpret_cast<t8 *>(out + to) = x;
    }
}

struct KeepArgs {
    f3s_cache_t c;
    const int32_t *table, *lens, *picks;
    int32_t *new_lens;
    int32_t max_pages, page_shift, n_new, n_picks;
    int32_t blocks;  // workgroups of a sequence
};

// Kept tokens of a sequence move towards its front, so that the i-th goes to a place at
// or before its own, and the later ones' own places lie behind it.  A thread has one
// 16-byte piece of a row (of one key head, of K or V) of every token and moves them in
// order, kAhead at a time, all loaded before the first is stored: no thread reads what
// another writes.  The places of a round of picks are looked up once, a thread each.
constexpr int kKeepAhead = 8;
constexpr int32_t kMostPicks = 1 << 30;  // (their indexes stay below 2^31)

__global__ __launch_bounds__(kThreads) void k_cache_keep(KeepArgs a)
{
    __shared__ int64_t s_from[kThreads], s_to[kThreads];  // in tokens of one head, or -1
    __shared__ int s_end;
    const int b = (int)blockIdx.x / a.blocks, part = (int)blockIdx.x - b * a.blocks;
    const int pieces = a.c.d / 16;
    const int f = part * kThreads + (int)threadIdx.x;
    const int head = f / (2 * pieces), side = f / pieces & 1, piece = f % pieces;
    const bool mine = head < a.c.n_kv_heads;
    uint8_t *const codes = reinterpret_cast<uint8_t *>(side ? a.c.v : a.c.k) + piece * 16;
    uint8_t *const powers = side ? a.c.v_exp : a.c.k_exp;
    const int32_t *const picks = a.picks + (int64_t)b * a.n_picks;
    const int32_t *const table = a.table + (int64_t)b * a.max_pages;
    const int64_t first = cache_position(a.lens[b], a.n_new, 0), front = first < 0 ? 0 : first;
    // row of the cache of a place
    auto row = [&](int64_t slot) {
        const int64_t page = slot >> a.page_shift;
        return ((page * a.c.n_kv_heads + head) << a.page_shift) +
               (slot & ((1 << a.page_shift) - 1));
    };
    int kept = 0;
    for (int at = 0; at < a.n_picks; at += kThreads) {
        const int i = at + (int)threadIdx.x;
        const int pick = i < a.n_picks ? picks[i] : -1;
        const int before = i < a.n_picks && i ? picks[i - 1] : -1;
        const bool ok = i < a.n_picks && pick > before && pick < a.n_new && first + pick >= 0;
        if (threadIdx.x == 0) s_end = kThreads;
        __syncthreads();
        if (!ok) atomicMin(&s_end, (int)threadIdx.x);
        int64_t from = -1, to = -1;
        if (ok) {
            from = cache_slot(table, a.max_pages, a.c.n_pages, a.page_shift, first + pick);
            to = cache_slot(table, a.max_pages, a.c.n_pages, a.page_shift, front + i);
            if (to == from || to < 0) from = -1;
        }
        s_from[threadIdx.x] = from;
        s_to[threadIdx.x] = to;
        __syncthreads();
        const int n = s_end;
        kept += n;
        for (int k0 = 0; mine && k0 < n; k0 += kKeepAhead) {
            u4 x[kKeepAhead];
            uint8_t e[kKeepAhead];
#pragma unroll
            for (int k = 0; k < kKeepAhead; ++k) {
                const int64_t slot = k0 + k < n ? s_from[k0 + k] : -1;
                if (slot < 0) continue;
                const int64_t r = row(slot);
                x[k] = *reinterpret_cast<const u4 *>(codes + r * a.c.d);
                if (piece == 0) e[k] = powers[r];
            }
#pragma unroll
            for (int k = 0; k < kKeepAhead; ++k) {
                if (k0 + k >= n || s_from[k0 + k] < 0) continue;
                const int64_t r = row(s_to[k0 + k]);
                *reinterpret_cast<u4 *>(codes + r * a.c.d) = x[k];
                if (piece == 0) powers[r] = e[k];
            }
        }
        if (n < kThreads) break;
        __syncthreads();  // (the places and the end are used up)
    }
    if (part == 0 && threadIdx.x == 0) a.new_lens[b] = (int32_t)(front + kept);
}

// The instance of F<D> for one of the feature sizes.
template <template <int> class F, typename... A>
hipError_t with_d(int d, A... args)
{
    switch (d) {
    case 32: return F<32>::launch(args...);
    case 64: return F<64>::launch(args...);
    case 96: return F<96>::launch(args...);
    case 128: return F<128>::launch(args...);
    case 160: return F<160>::launch(args...);
    case 192: return F<192>::launch(args...);
    case 224: return F<224>::launch(args...);
    default: return F<256>::launch(args...);
    }
}

template <int D>
struct Write {
    static hipError_t launch(const RowArgs &a, const void *K, const void *V, bool bf16,
                             hipStream_t s)
    {
        constexpr uint32_t per = kThreads / lanes_of(D);
        const uint32_t grid = (a.rows + per - 1) / per;
        if (bf16)
            k_cache_write<D, __bf16><<<grid, kThreads, 0, s>>>(a, (const __bf16 *)K,
                                                               (const __bf16 *)V);
        else
            k_cache_write<D, _Float16><<<grid, kThreads, 0, s>>>(a, (const _Float16 *)K,
                                                                 (const _Float16 *)V);
        return hipGetLastError();
    }
};

template <int D>
struct Read {
    static hipError_t launch(const RowArgs &a, void *K, void *V, f3s_dtype_t t, hipStream_t s)
    {
        constexpr uint32_t per = kThreads / lanes_of(D);
        const uint32_t grid = (a.rows + per - 1) / per;
        if (t == F3S_DTYPE_BF16)
            k_cache_read<D, __bf16><<<grid, kThreads, 0, s>>>(a, (__bf16 *)K, (__bf16 *)V);
        else if (t == F3S_DTYPE_F16)
            k_cache_read<D, _Float16><<<grid, kThreads, 0, s>>>(a, (_Float16 *)K,
                                                                (_Float16 *)V);
        else
            k_cache_read<D, float><<<grid, kThreads, 0, s>>>(a, (float *)K, (float *)V);
        return hipGetLastError();
    }
};

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && na && nb && x < y + nb && y < x + na;
}

// Whether n bytes at p share any with the cache or, where they are written
// (`out`), with what is read beside it.
bool meets(const void *p, size_t n, const RowArgs &a, bool out)
{
    const size_t places = (size_t)a.c.n_pages * a.c.n_kv_heads * a.c.page_size;
    const size_t seqs = a.rows / ((size_t)a.n_new * a.c.n_kv_heads);
    const struct {
        const void *p;
        size_t n;
    } with[] = {{a.c.k, places * a.c.d}, {a.c.v, places * a.c.d}, {a.c.k_exp, places},
                {a.c.v_exp, places}, {a.table, out ? seqs * a.max_pages * 4 : 0},
                {a.lens, out ? seqs * 4 : 0}};
    for (const auto &w : with)
        if (overlap(p, n, w.p, w.n)) return true;
    return false;
}

// Whether rows that are written to the cache would be written over others, some of
// its parts sharing memory.  (One place for K and V may get the same rows twice.)
bool folded(const f3s_cache_t &c, bool same_rows)
{
    const size_t places = (size_t)c.n_pages * c.n_kv_heads * c.page_size;
    const size_t codes = places * c.d;
    if (overlap(c.k, codes, c.k_exp, places) || overlap(c.v, codes, c.k_exp, places) ||
        overlap(c.k, codes, c.v_exp, places) || overlap(c.v, codes, c.v_exp, places))
        return true;
    if (same_rows && c.k == c.v && c.k_exp == c.v_exp) return false;
    return overlap(c.k, codes, c.v, codes) || overlap(c.k_exp, places, c.v_exp, places);
}

}  // namespace

f3s_status_t check_cache(const f3s_cache_t *c)
{
    if (!c) return F3S_ERR_INVALID_VALUE;
    if (c->d < 32 || c->d > kMaxD || c->d % 32 != 0) return F3S_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        return F3S_ERR_UNSUPPORTED;
    if (c->n_pages < 1 || c->n_kv_heads < 1) return F3S_ERR_INVALID_VALUE;
    if (!c->k || !c->v || !c->k_exp || !c->v_exp || !aligned(c->k, 16) || !aligned(c->v, 16) ||
        !aligned(c->k_exp, 16) || !aligned(c->v_exp, 16))
        return F3S_ERR_INVALID_VALUE;
    return F3S_OK;
}

}  // namespace f3s

namespace {

// The checks that writing and reading share; F3S_OK with a->rows = 0: nothing to do.
f3s_status_t row_args(const f3s_cache_t *c, const int32_t *table, int32_t max_pages,
                      const int32_t *lens, int32_t n_seqs, int32_t n_new, f3s::RowArgs *a)
{
    if (f3s_status_t st = f3s::check_cache(c)) return st;
    if (n_seqs < 0 || n_new < 0 || max_pages < 0) return F3S_ERR_INVALID_VALUE;
    a->rows = 0;
    if (n_seqs == 0 || n_new == 0) return F3S_OK;
    if (!lens || !f3s::aligned(lens, 4) || (max_pages && !table) || !f3s::aligned(table, 4))
        return F3S_ERR_INVALID_VALUE;
    if ((double)n_seqs * n_new * c->n_kv_heads >
        (double)f3s::kMostGrid * (f3s::kThreads / f3s::lanes_of(c->d)))
        return F3S_ERR_TOO_LARGE;
    *a = f3s::RowArgs{*c, table, lens, max_pages, __builtin_ctz(c->page_size), n_new,
                      (uint32_t)n_seqs * (uint32_t)n_new * (uint32_t)c->n_kv_heads};
    return F3S_OK;
}

}  // namespace

extern "C" {

f3s_status_t f3s_cache_write(const f3s_cache_t *cache, const void *K, const void *V,
                             f3s_dtype_t dtype, const int32_t *table, int32_t max_pages,
                             const int32_t *lens, int32_t n_seqs, int32_t n_new,
                             hipStream_t stream)
{
    f3s::RowArgs a;
    if (f3s_status_t st = row_args(cache, table, max_pages, lens, n_seqs, n_new, &a))
        return f3s::set_status(st);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return f3s::set_status(F3S_ERR_UNSUPPORTED);
    if (a.rows == 0) return F3S_OK;
    const size_t bytes = (size_t)a.rows * cache->d * 2;
    if (!K || !V || !f3s::aligned(K, 16) || !f3s::aligned(V, 16) || f3s::folded(*cache, K == V) ||
        f3s::meets(K, bytes, a, false) || f3s::meets(V, bytes, a, false))
        return f3s::set_status(F3S_ERR_INVALID_VALUE);
    return f3s::set_status(f3s::status_of(
        f3s::with_d<f3s::Write>(cache->d, a, K, V, dtype == F3S_DTYPE_BF16, stream)));
}

f3s_status_t f3s_cache_read(const f3s_cache_t *cache, void *K, void *V, f3s_dtype_t dtype,
                            const int32_t *table, int32_t max_pages, const int32_t *lens,
                            int32_t n_seqs, int32_t n_new, hipStream_t stream)
{
    f3s::RowArgs a;
    if (f3s_status_t st = row_args(cache, table, max_pages, lens, n_seqs, n_new, &a))
        return f3s::set_status(st);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16 && dtype != F3S_DTYPE_F32)
        return f3s::set_status(F3S_ERR_UNSUPPORTED);
    if (a.rows == 0 || (!K && !V)) return F3S_OK;
    const size_t bytes = (size_t)a.rows * cache->d * (dtype == F3S_DTYPE_F32 ? 4 : 2);
    if (!f3s::aligned(K, 16) || !f3s::aligned(V, 16) || f3s::meets(K, bytes, a, true) ||
        f3s::meets(V, bytes, a, true) || f3s::overlap(K, bytes, V, bytes))
        return f3s::set_status(F3S_ERR_INVALID_VALUE);
    return f3s::set_status(
        f3s::status_of(f3s::with_d<f3s::Read>(cache->d, a, K, V, dtype, stream)));
}

f3s_status_t f3s_cache_keep(const f3s_cache_t *cache, const int32_t *table, int32_t max_pages,
                            const int32_t *lens, int32_t n_seqs, int32_t n_new,
                            const int32_t *picks, int32_t n_picks, int32_t *new_lens,
                            hipStream_t stream)
{
    using f3s::overlap;
    if (f3s_status_t st = f3s::check_cache(cache)) return f3s::set_status(st);
    if (n_seqs < 0 || n_new < 0 || n_picks < 0 || max_pages < 0)
        return f3s::set_status(F3S_ERR_INVALID_VALUE);
    if (n_seqs == 0) return F3S_OK;
    if (!lens || !new_lens || (max_pages && !table) || (n_picks && !picks) ||
        !f3s::aligned(lens, 4) || !f3s::aligned(new_lens, 4) || !f3s::aligned(table, 4) ||
        !f3s::aligned(picks, 4) || f3s::folded(*cache, false))
        return f3s::set_status(F3S_ERR_INVALID_VALUE);
    if (n_picks > f3s::kMostPicks) return f3s::set_status(F3S_ERR_TOO_LARGE);
    const int64_t threads = (int64_t)cache->n_kv_heads * (cache->d / 8);
    const int64_t blocks = (threads + f3s::kThreads - 1) / f3s::kThreads;
    if ((double)blocks * n_seqs > (double)f3s::kMostGrid || threads > 0x7FFFFFFF - f3s::kThreads)
        return f3s::set_status(F3S_ERR_TOO_LARGE);
    const size_t places = (size_t)cache->n_pages * cache->n_kv_heads * cache->page_size;
    const size_t lb = (size_t)n_seqs * 4;
    const struct {
        const void *p;
        size_t n;
    } parts[] = {{cache->k, places * cache->d}, {cache->v, places * cache->d},
                 {cache->k_exp, places}, {cache->v_exp, places}},
      read[] = {{table, lb * max_pages}, {lens, lb}, {picks, lb * n_picks}};
    for (const auto &y : read) {
        if (overlap(new_lens, lb, y.p, y.n)) return f3s::set_status(F3S_ERR_INVALID_VALUE);
        for (const auto &x : parts)
            if (overlap(x.p, x.n, y.p, y.n)) return f3s::set_status(F3S_ERR_INVALID_VALUE);
    }
    for (const auto &x : parts)
        if (overlap(x.p, x.n, new_lens, lb)) return f3s::set_status(F3S_ERR_INVALID_VALUE);
    const f3s::KeepArgs a = {*cache, table, lens, picks, new_lens, max_pages,
                             __builtin_ctz(cache->page_size), n_new, n_picks, (int32_t)blocks};
    f3s::k_cache_keep<<<(unsigned)(blocks * n_seqs), f3s::kThreads, 0, stream>>>(a);
    return f3s::set_status(f3s::status_of(hipGetLastError()));
}

}  // extern "C"
