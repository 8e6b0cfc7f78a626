// f3s_cross_plan, f3s_cross_forward, f3s_cross_backward: the division of a
// ragged batch among workgroups, checks, workspace.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <memory>
#include <new>
#include <vector>

#include "cross_backward.h"
#include "cross_few.h"
#include "dense_division.h"

namespace {

using f3s::DenseItem;
using f3s::DenseMerge;
using f3s::Division;
using f3s::Range;
using f3s::set_status;

constexpr int64_t kUnits = 256;  // compute units
// Workgroups that the kernel of few rows aims at.
constexpr int64_t kFewWorkgroups = 4 * kUnits;
// What a launch that joins pieces costs there, in units of 64 keys, of which one
// takes 0.4 us (d = 64) to 0.6 us (128).  One token of 4 sequences over 500 to 1,000
// keys, 8 key heads, whole and in pieces: 8.0 and 6.7 us on the GPU and 9.2 and
// 13.5 us from one call to the next (d = 64), 12.0 and 7.9, 12.1 and 13.4 (128).
constexpr double kFewLaunch = 10;
// Query rows of a key head up to which the forward takes the kernel of few rows:
// one sequence's row over 100 keys takes 2.7 us with it and 3.8 with the other, 4
// over 8,192 keys 8.6 and 10.8; 16 rows of 16 sequences over 2,048 keys 28.9 and
// 26.7 (8 key heads of 128 in the last two).
constexpr int64_t kFewLongest = 8;

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }
bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na && nb && x < y + nb && y < x + na;
}

f3s_cross_plan_t make_plan(const int32_t *q_ptr, const int32_t *k_ptr, const int32_t *q_len,
                           const int32_t *k_len, int32_t n, int32_t n_heads, int32_t n_kv,
                           int32_t d, f3s_status_t *st)
{
    *st = F3S_ERR_INVALID_VALUE;
    if (!q_ptr || !k_ptr || n < 0 || n_kv < 1 || n_heads < 1 || n_heads % n_kv) return nullptr;
    // (a tile's 64 rows of all heads have to lie within 4 GiB)
    if (d < 32 || d > f3s::kMaxD || d % 32 != 0 || n_heads > 65535) {
        *st = F3S_ERR_UNSUPPORTED;
        return nullptr;
    }
    if (q_ptr[0] != 0 || k_ptr[0] != 0) return nullptr;
    const int64_t g = n_heads / n_kv;
    std::vector<Range> fwd, keys;
    int64_t longest = 0;
    for (int32_t b = 0; b < n; ++b) {
        if (q_ptr[b + 1] < q_ptr[b] || k_ptr[b + 1] < k_ptr[b]) return nullptr;
        const int64_t q = q_ptr[b + 1] - (int64_t)q_ptr[b], k = k_ptr[b + 1] - (int64_t)k_ptr[b];
        const int64_t ql = q_len ? q_len[b] : q, kl = k_len ? k_len[b] : k;
        if (ql < 0 || ql > q || kl < 0 || kl > k) return nullptr;
        // (rows that are padding walk nothing: their results are zeros)
        if (ql) fwd.push_back({q_ptr[b] * g, ql * g, k_ptr[b], kl});
        if (ql < q) fwd.push_back({(q_ptr[b] + ql) * g, (q - ql) * g, 0, 0});
        if (kl) keys.push_back({k_ptr[b], kl, q_ptr[b] * g, ql * g});
        if (kl < k) keys.push_back({k_ptr[b] + kl, k - kl, 0, 0});
        if (ql * g > longest) longest = ql * g;
    }
    *st = F3S_ERR_TOO_LARGE;
    // (a row's number and a tile add up to less than 2^31)
    if (q_ptr[n] * g > 0x7FFFF000 || k_ptr[n] > 0x7FFFF000 ||
        (double)q_ptr[n] * n_heads / 16 + n_heads > 2147483647.0)
        return nullptr;
    Division f, dq, dkv;
    const char *rows_env = getenv("F3S_CROSS_ROWS");
    const bool few = rows_env && *rows_env ? atoi(rows_env) == f3s::kFewRows
                                           : longest <= kFewLongest;
    if (few)
        f.make(fwd, n_kv, f3s::kFewRows, 64, 256, kFewWorkgroups, kFewLaunch);
    else
        f.make(fwd, n_kv, f3s::kManyRows, 64, 256, kUnits * f3s::many_waves(d));
    dq.make(fwd, n_kv, f3s::kManyRows, 64, 256, kUnits * f3s::dq_waves(d));
    dkv.make(keys, n_kv, f3s::kManyRows, 64, 256,
             kUnits * f3s::dkv_waves(d) / f3s::dkv_halves(d));
    if (!f.fits() || !dq.fits() || !dkv.fits()) return nullptr;

    std::unique_ptr<f3s_cross_plan_s, void (*)(f3s_cross_plan_t)> p(new f3s_cross_plan_s,
                                                                    f3s_cross_destroy);
    p->n_heads = n_heads;
    p->n_kv = n_kv;
    p->g = (int32_t)g;
    p->d = d;
    p->q_rows = q_ptr[n];
    p->k_rows = k_ptr[n];
    p->few = few;
    p->n_fwd = (int32_t)f.items.size();
    p->n_fwd_merge = (int32_t)f.merges.size();
    p->fwd_merge_rows = f.merge_rows;
    p->fwd_parts = f.parts;
    p->n_dq = (int32_t)dq.items.size();
    p->n_dq_merge = (int32_t)dq.merges.size();
    p->dq_merge_rows = dq.merge_rows;
    p->dq_parts = dq.parts;
    p->n_dkv = (int32_t)dkv.items.size();
    p->n_dkv_merge = (int32_t)dkv.merges.size();
    p->dkv_merge_rows = dkv.merge_rows;
    p->dkv_parts = dkv.parts;
    const struct {
        const void *src;
        size_t bytes;
        void **dst;
    } lists[] = {
        {f.items.data(), f.items.size() * sizeof(DenseItem), (void **)&p->fwd},
        {f.merges.data(), f.merges.size() * sizeof(DenseMerge), (void **)&p->fwd_merge},
        {dq.items.data(), dq.items.size() * sizeof(DenseItem), (void **)&p->dq},
        {dq.merges.data(), dq.merges.size() * sizeof(DenseMerge), (void **)&p->dq_merge},
        {dkv.items.data(), dkv.items.size() * sizeof(DenseItem), (void **)&p->dkv},
        {dkv.merges.data(), dkv.merges.size() * sizeof(DenseMerge), (void **)&p->dkv_merge},
    };
    size_t bytes = 0;
    for (const auto &l : lists) bytes += round256(l.bytes);
    std::vector<char> host(bytes);
    hipError_t e = hipGetDevice(&p->device);
    if (e == hipSuccess && bytes) e = f3s::limited_malloc(&p->store, bytes);
    if (e == hipSuccess && bytes) {
        size_t at = 0;
        for (const auto &l : lists) {
            if (l.bytes) memcpy(host.data() + at, l.src, l.bytes);
            *l.dst = (char *)p->store + at;
            at += round256(l.bytes);
        }
        e = hipMemcpy(p->store, host.data(), bytes, hipMemcpyHostToDevice);
    }
    *st = f3s::status_of(e);
    return e == hipSuccess ? p.release() : nullptr;
}

bool on_device(const f3s_cross_plan_s *p, hipStream_t stream)
{
    int dev = -1;
    const hipError_t e = stream ? hipStreamGetDevice(stream, &dev) : hipGetDevice(&dev);
    return e == hipSuccess && dev == p->device;
}

// Partial rows of d floats, then their records of `record` floats.
size_t parts_bytes(int64_t rows, int32_t d, int32_t record)
{
    return rows ? round256((size_t)rows * d * 4) + round256((size_t)rows * record * 4) : 0;
}

// |scale| log2 e.  Scores that are left out are -inf and stay so under a factor
// that is not 0: a scale of 0 counts as 2^-120, which turns every finite score
// of an f16 or bf16 product below 2^100 into 0 as well.
float base2_scale(float scale)
{
    const float s = f3s::scale_log2e(scale);
    return s < 0x1p-120f ? 0x1p-120f : s;
}

bool workspace_ok(const void *w, size_t have, size_t need)
{
    return need == 0 || (w && aligned(w, 256) && have >= need);
}

}  // namespace

extern "C" {

f3s_cross_plan_t f3s_cross_plan(const int32_t *q_ptr, const int32_t *k_ptr,
                                const int32_t *q_len, const int32_t *k_len, int32_t n_seqs,
                                int32_t n_heads, int32_t n_kv_heads, int32_t d)
{
    f3s_status_t st;
    f3s_cross_plan_t p = nullptr;
    try {
        p = make_plan(q_ptr, k_ptr, q_len, k_len, n_seqs, n_heads, n_kv_heads, d, &st);
    } catch (...) {  // (std::bad_alloc, std::length_error)
        st = F3S_ERR_OUT_OF_MEMORY;
    }
    set_status(st);
    return p;
}

void f3s_cross_destroy(f3s_cross_plan_t p)
{
    if (!p) return;
    if (p->store) (void)hipFree(p->store);
    delete p;
}

size_t f3s_cross_forward_workspace_bytes(f3s_cross_plan_t p)
{
    return p ? parts_bytes(p->fwd_parts, p->d, 2) : 0;
}

f3s_status_t f3s_cross_forward(f3s_cross_plan_t p, const void *Q, const void *K,
                               const void *V, f3s_dtype_t dtype, void *O, float *lse,
                               float scale, void *workspace, size_t workspace_bytes,
                               hipStream_t stream)
{
    if (!p || !isfinite(scale)) return set_status(F3S_ERR_INVALID_VALUE);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return set_status(F3S_ERR_UNSUPPORTED);
    if (p->q_rows == 0) return F3S_OK;
    if (!on_device(p, stream)) return set_status(F3S_ERR_INVALID_VALUE);
    if (!Q || !O || !lse || (p->k_rows && (!K || !V)) || !aligned(Q, 16) || !aligned(K, 16) ||
        !aligned(V, 16) || !aligned(O, 16) || !aligned(lse, 4))
        return set_status(F3S_ERR_INVALID_VALUE);
    const size_t need = f3s_cross_forward_workspace_bytes(p);
    if (!workspace_ok(workspace, workspace_bytes, need))
        return set_status(F3S_ERR_INVALID_VALUE);
    const size_t qb = (size_t)p->q_rows * p->n_heads * p->d * 2;
    const size_t kb = (size_t)p->k_rows * p->n_kv * p->d * 2;
    const size_t lb = (size_t)p->q_rows * p->n_heads * 4;
    const struct {
        const void *p;
        size_t n;
    } in[] = {{Q, qb}, {K, kb}, {V, kb}};
    for (const auto &x : in)
        if (overlaps(O, qb, x.p, x.n) || overlaps(lse, lb, x.p, x.n) ||
            overlaps(workspace, need, x.p, x.n))
            return set_status(F3S_ERR_INVALID_VALUE);
    if (overlaps(O, qb, lse, lb) || overlaps(O, qb, workspace, need) ||
        overlaps(lse, lb, workspace, need))
        return set_status(F3S_ERR_INVALID_VALUE);
    f3s::FewArgs a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.O = O;
    a.lse = lse;
    a.q = f3s::query_rows(p->n_heads, p->g);
    a.n_kv = p->n_kv;
    a.sl2 = base2_scale(scale);
    a.flip = signbit(scale) ? 0x80008000u : 0u;
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + round256((size_t)p->fwd_parts * p->d * 4));
    const bool bf16 = dtype == F3S_DTYPE_BF16;
    auto launch = p->few ? (bf16 ? f3s::launch_cross_few_bf16 : f3s::launch_cross_few_f16)
                         : (bf16 ? f3s::launch_cross_many_bf16 : f3s::launch_cross_many_f16);
    hipError_t e = launch(*p, a, stream);
    if (e == hipSuccess && p->n_fwd_merge) {
        const f3s::CrossMergeArgs m = {p->fwd_merge, a.part_o, a.part_ml, O, lse, a.q, 0};
        e = bf16 ? f3s::launch_cross_merge_bf16(*p, m, stream)
                 : f3s::launch_cross_merge_f16(*p, m, stream);
    }
    return set_status(f3s::status_of(e));
}

size_t f3s_cross_backward_workspace_bytes(f3s_cross_plan_t p)
{
    if (!p) return 0;
    return round256((size_t)p->q_rows * p->n_heads * 8) + parts_bytes(p->dq_parts, p->d, 0) +
           parts_bytes(p->dkv_parts, 2 * p->d, 0);
}

f3s_status_t f3s_cross_backward(f3s_cross_plan_t p, const void *Q, const void *K,
                                const void *V, f3s_dtype_t dtype, const void *O,
                                const void *dO, const float *lse, void *dQ, void *dK,
                                void *dV, float scale, void *workspace,
                                size_t workspace_bytes, hipStream_t stream)
{
    if (!p || !isfinite(scale)) return set_status(F3S_ERR_INVALID_VALUE);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return set_status(F3S_ERR_UNSUPPORTED);
    if (p->q_rows == 0 && p->k_rows == 0) return F3S_OK;
    if (!on_device(p, stream)) return set_status(F3S_ERR_INVALID_VALUE);
    const size_t qb = (size_t)p->q_rows * p->n_heads * p->d * 2;
    const size_t kb = (size_t)p->k_rows * p->n_kv * p->d * 2;
    const size_t lb = (size_t)p->q_rows * p->n_heads * 4;
    const size_t need = f3s_cross_backward_workspace_bytes(p);
    if (!workspace_ok(workspace, workspace_bytes, need))
        return set_status(F3S_ERR_INVALID_VALUE);
    struct Span {
        const void *p;
        size_t n;
    };
    const Span in[] = {{Q, qb}, {K, kb}, {V, kb}, {O, qb}, {dO, qb}, {lse, lb},
                       {workspace, need}};
    const Span out[] = {{dQ, qb}, {dK, kb}, {dV, kb}};
    const Span &stats = in[5], &room = in[6];
    for (const Span &x : in)
        if ((x.n && !x.p) || !aligned(x.p, &x == &stats ? 4 : 16) ||
            (&x != &room && overlaps(room.p, room.n, x.p, x.n)))
            return set_status(F3S_ERR_INVALID_VALUE);
    for (const Span &x : out) {
        if ((x.n && !x.p) || !aligned(x.p, 16)) return set_status(F3S_ERR_INVALID_VALUE);
        for (const Span &y : in)
            if (overlaps(x.p, x.n, y.p, y.n)) return set_status(F3S_ERR_INVALID_VALUE);
        for (const Span &y : out)
            if (&x != &y && overlaps(x.p, x.n, y.p, y.n))
                return set_status(F3S_ERR_INVALID_VALUE);
    }
    f3s::CrossBwdArgs a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.O = O;
    a.G = dO;
    a.lse = lse;
    a.dQ = dQ;
    a.dK = dK;
    a.dV = dV;
    a.q = f3s::query_rows(p->n_heads, p->g);
    a.n_kv = p->n_kv;
    a.sl2 = base2_scale(scale);
    a.scale = scale;
    a.flip = signbit(scale) ? 0x80008000u : 0u;
    char *w = (char *)workspace;
    a.stats = (float2 *)w;
    w += round256((size_t)p->q_rows * p->n_heads * 8);
    a.part_dq = (float *)w;
    w += parts_bytes(p->dq_parts, p->d, 0);
    a.part_dkv = (float *)w;
    return set_status(f3s::status_of(dtype == F3S_DTYPE_BF16
                                         ? f3s::launch_cross_backward_bf16(*p, a, stream)
                                         : f3s::launch_cross_backward_f16(*p, a, stream)));
}

}  // extern "C"
