// f3s_cross_plan, f3s_cross_forward, f3s_cross_backward: the division of a
// ragged batch among workgroups, checks, workspace.
#include <stdlib.h>

#include <memory>
#include <new>
#include <vector>

#include "dense_host.h"

namespace {

using f3s::DenseItem;
using f3s::DenseMerge;
using f3s::Division;
using f3s::Range;
using f3s::set_status;

// Workgroups that the kernel of few rows aims at.
constexpr int64_t kFewWorkgroups = 4 * f3s::kUnits;
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
        f.make(fwd, n_kv, f3s::kManyRows, 64, 256, f3s::kUnits * f3s::many_waves(d));
    dq.make(fwd, n_kv, f3s::kManyRows, 64, 256, f3s::kUnits * f3s::dq_waves(d));
    dkv.make(keys, n_kv, f3s::kManyRows, 64, 256,
             f3s::kUnits * f3s::dkv_waves(d) / f3s::dkv_halves(d));
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
    f3s::set_divisions(p.get(), f, dq, dkv);
    const f3s::PlanList lists[] = {
        {f.items.data(), f.items.size() * sizeof(DenseItem), (void **)&p->fwd},
        {f.merges.data(), f.merges.size() * sizeof(DenseMerge), (void **)&p->fwd_merge},
        {dq.items.data(), dq.items.size() * sizeof(DenseItem), (void **)&p->dq},
        {dq.merges.data(), dq.merges.size() * sizeof(DenseMerge), (void **)&p->dq_merge},
        {dkv.items.data(), dkv.items.size() * sizeof(DenseItem), (void **)&p->dkv},
        {dkv.merges.data(), dkv.merges.size() * sizeof(DenseMerge), (void **)&p->dkv_merge},
    };
    const hipError_t e = f3s::store_lists(p.get(), lists, sizeof lists / sizeof *lists);
    *st = f3s::status_of(e);
    return e == hipSuccess ? p.release() : nullptr;
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
    return f3s::forward_workspace(p);
}

f3s_status_t f3s_cross_forward(f3s_cross_plan_t p, const void *Q, const void *K,
                               const void *V, f3s_dtype_t dtype, void *O, float *lse,
                               float scale, void *workspace, size_t workspace_bytes,
                               hipStream_t stream)
{
    return f3s::dense_forward(
        p, Q, K, V, dtype, O, lse, scale, workspace, workspace_bytes, stream,
        [&](const f3s::FewArgs &a, bool bf16) {
            if (p->few)
                return bf16 ? f3s::launch_cross_few_bf16(*p, a, stream)
                            : f3s::launch_cross_few_f16(*p, a, stream);
            return bf16 ? f3s::launch_cross_many_bf16(*p, a, stream)
                        : f3s::launch_cross_many_f16(*p, a, stream);
        });
}

size_t f3s_cross_backward_workspace_bytes(f3s_cross_plan_t p)
{
    return f3s::backward_workspace(p);
}

f3s_status_t f3s_cross_backward(f3s_cross_plan_t p, const void *Q, const void *K,
                                const void *V, f3s_dtype_t dtype, const void *O,
                                const void *dO, const float *lse, void *dQ, void *dK,
                                void *dV, float scale, void *workspace,
                                size_t workspace_bytes, hipStream_t stream)
{
    return f3s::dense_backward(p, Q, K, V, dtype, O, dO, lse, dQ, dK, dV, scale, workspace,
                               workspace_bytes, stream,
                               [&](const f3s::CrossBwdArgs &a, bool bf16) {
                                   return bf16 ? f3s::launch_cross_backward_bf16(*p, a, stream)
                                               : f3s::launch_cross_backward_f16(*p, a, stream);
                               });
}

}  // extern "C"
