// f3s_window_plan, f3s_window_forward, f3s_window_backward: the division of a ragged
// batch among workgroups.
#include <memory>
#include <new>
#include <vector>

#include "dense_host.h"
#include "window.h"
#include "window_ranges.h"

namespace {

using f3s::DenseItem;
using f3s::DenseMerge;
using f3s::Division;
using f3s::set_status;
using f3s::WindowItem;
using f3s::WindowRule;

// Largest window and number of sinks (a larger one is this one: positions are below
// 2^31).
constexpr int32_t kMostWindow = 1 << 30;

std::vector<WindowItem> window_items(const Division &d, const std::vector<f3s::WindowShared> &shared)
{
    std::vector<WindowItem> out(d.items.size());
    for (size_t i = 0; i < out.size(); ++i) {
        static_cast<DenseItem &>(out[i]) = d.items[i];
        const f3s::WindowShared &s = shared[d.items[i].tag];
        out[i].key0 = s.key0;
        out[i].shift = s.shift;
        out[i].keys = s.keys;
    }
    return out;
}

f3s_window_plan_t make_plan(const int32_t *q_ptr, const int32_t *k_ptr, const int32_t *q_len,
                            const int32_t *k_len, int32_t n, int32_t n_heads, int32_t n_kv,
                            int32_t d, int32_t window, int32_t sinks, f3s_status_t *st)
{
    *st = F3S_ERR_INVALID_VALUE;
    if (!q_ptr || !k_ptr || n < 0 || n_kv < 1 || n_heads < 1 || n_heads % n_kv || window < 0 ||
        sinks < 0)
        return nullptr;
    // (a tile's 64 rows of all heads have to lie within 4 GiB)
    if (d < 32 || d > f3s::kMaxD || d % 32 != 0 || n_heads > 65535) {
        *st = F3S_ERR_UNSUPPORTED;
        return nullptr;
    }
    if (q_ptr[0] != 0 || k_ptr[0] != 0) return nullptr;
    const WindowRule rule = {std::min(window, kMostWindow), std::min(sinks, kMostWindow)};
    const int64_t g = n_heads / n_kv, tile = f3s::kWindowTile;
    static_assert(f3s::kWindowTile == f3s::kManyRows, "");
    double q_tiles = 0, k_tiles = 0;
    for (int32_t b = 0; b < n; ++b) {
        if (q_ptr[b + 1] < q_ptr[b] || k_ptr[b + 1] < k_ptr[b]) return nullptr;
        const int64_t q = q_ptr[b + 1] - (int64_t)q_ptr[b], k = k_ptr[b + 1] - (int64_t)k_ptr[b];
        const int64_t ql = q_len ? q_len[b] : q, kl = k_len ? k_len[b] : k;
        if (ql < 0 || ql > q || kl < 0 || kl > k) return nullptr;
        q_tiles += (double)(f3s::ceil_div(ql * g, tile) + f3s::ceil_div((q - ql) * g, tile));
        // (the sinks' tiles are their own)
        k_tiles += (double)(f3s::ceil_div(kl, tile) + f3s::ceil_div(k - kl, tile)) +
                   (sinks && window < kl ? 1 : 0);
    }
    *st = F3S_ERR_TOO_LARGE;
    // (a row's number and a tile add up to less than 2^31)
    if (q_ptr[n] * g > 0x7FFFF000 || k_ptr[n] > 0x7FFFF000 ||
        (double)q_ptr[n] * n_heads / 16 + n_heads > 2147483647.0 ||
        std::max(q_tiles, k_tiles) * n_kv > Division::kMostTiles)
        return nullptr;
    const f3s::WindowRanges r = f3s::window_ranges(q_ptr, k_ptr, q_len, k_len, n, g, rule);
    Division f, dq, dkv;
    f.make(r.queries, n_kv, tile, f3s::kWindowUnit, 256, f3s::kUnits * f3s::many_waves(d));
    dq.make(r.queries, n_kv, tile, f3s::kWindowUnit, 256, f3s::kUnits * f3s::dq_waves(d));
    dkv.make(r.keys, n_kv, tile, 64, 256, f3s::kUnits * f3s::dkv_waves(d) / f3s::dkv_halves(d),
             Division::kLaunch, true);
    if (!f.fits() || !dq.fits() || !dkv.fits()) return nullptr;

    std::unique_ptr<f3s_window_plan_s, void (*)(f3s_window_plan_t)> p(new f3s_window_plan_s,
                                                                      f3s_window_destroy);
    p->n_heads = n_heads;
    p->n_kv = n_kv;
    p->g = (int32_t)g;
    p->d = d;
    p->q_rows = q_ptr[n];
    p->k_rows = k_ptr[n];
    p->rule = rule;
    f3s::set_divisions(p.get(), f, dq, dkv);
    const std::vector<WindowItem> fi = window_items(f, r.shared),
                                  qi = window_items(dq, r.shared),
                                  ki = window_items(dkv, r.shared);
    const f3s::PlanList lists[] = {
        {fi.data(), fi.size() * sizeof(WindowItem), (void **)&p->window_fwd},
        {f.merges.data(), f.merges.size() * sizeof(DenseMerge), (void **)&p->fwd_merge},
        {qi.data(), qi.size() * sizeof(WindowItem), (void **)&p->window_dq},
        {dq.merges.data(), dq.merges.size() * sizeof(DenseMerge), (void **)&p->dq_merge},
        {ki.data(), ki.size() * sizeof(WindowItem), (void **)&p->window_dkv},
        {dkv.merges.data(), dkv.merges.size() * sizeof(DenseMerge), (void **)&p->dkv_merge},
    };
    const hipError_t e = f3s::store_lists(p.get(), lists, sizeof lists / sizeof *lists);
    *st = f3s::status_of(e);
    return e == hipSuccess ? p.release() : nullptr;
}

}  // namespace

extern "C" {

f3s_window_plan_t f3s_window_plan(const int32_t *q_ptr, const int32_t *k_ptr,
                                  const int32_t *q_len, const int32_t *k_len, int32_t n_seqs,
                                  int32_t n_heads, int32_t n_kv_heads, int32_t d,
                                  int32_t window, int32_t sinks)
{
    f3s_status_t st;
    f3s_window_plan_t p = nullptr;
    try {
        p = make_plan(q_ptr, k_ptr, q_len, k_len, n_seqs, n_heads, n_kv_heads, d, window, sinks,
                      &st);
    } catch (...) {  // (std::bad_alloc, std::length_error)
        st = F3S_ERR_OUT_OF_MEMORY;
    }
    set_status(st);
    return p;
}

void f3s_window_destroy(f3s_window_plan_t p)
{
    if (!p) return;
    if (p->store) (void)hipFree(p->store);
    delete p;
}

size_t f3s_window_forward_workspace_bytes(f3s_window_plan_t p)
{
    return f3s::forward_workspace(p);
}

f3s_status_t f3s_window_forward(f3s_window_plan_t p, const void *Q, const void *K,
                                const void *V, f3s_dtype_t dtype, void *O, float *lse,
                                float scale, void *workspace, size_t workspace_bytes,
                                hipStream_t stream)
{
    return f3s::dense_forward(p, Q, K, V, dtype, O, lse, scale, workspace, workspace_bytes,
                              stream, [&](const f3s::FewArgs &a, bool bf16) {
                                  return bf16 ? f3s::launch_window_bf16(*p, a, stream)
                                              : f3s::launch_window_f16(*p, a, stream);
                              });
}

size_t f3s_window_backward_workspace_bytes(f3s_window_plan_t p)
{
    return f3s::backward_workspace(p);
}

f3s_status_t f3s_window_backward(f3s_window_plan_t p, const void *Q, const void *K,
                                 const void *V, f3s_dtype_t dtype, const void *O,
                                 const void *dO, const float *lse, void *dQ, void *dK,
                                 void *dV, float scale, void *workspace,
                                 size_t workspace_bytes, hipStream_t stream)
{
    return f3s::dense_backward(p, Q, K, V, dtype, O, dO, lse, dQ, dK, dV, scale, workspace,
                               workspace_bytes, stream,
                               [&](const f3s::CrossBwdArgs &a, bool bf16) {
                                   return bf16 ? f3s::launch_window_backward_bf16(*p, a, stream)
                                               : f3s::launch_window_backward_f16(*p, a, stream);
                               });
}

}  // extern "C"
