// Host side that cross attention (cross.hip) and window attention (window.hip) share: a
// plan's lists, the checks of a forward and a backward call, and their arguments.
#pragma once

#include <math.h>
#include <string.h>

#include <vector>

#include "cross_backward.h"
#include "cross_few.h"
#include "dense_division.h"

namespace f3s {

constexpr int64_t kUnits = 256;  // compute units

inline size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }
inline bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na && nb && x < y + nb && y < x + na;
}

// The divisions' numbers in a plan.
inline void set_divisions(f3s_cross_plan_s *p, const Division &f, const Division &dq,
                          const Division &dkv)
{
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
}

// A list on the host, and where a plan keeps the address of its copy.
struct PlanList {
    const void *src;
    size_t bytes;
    void **dst;
};

// Copies the lists into one allocation of the plan's, on the current device.
inline hipError_t store_lists(f3s_cross_plan_s *p, const PlanList *lists, size_t n)
{
    size_t bytes = 0;
    for (size_t i = 0; i < n; ++i) bytes += round256(lists[i].bytes);
    std::vector<char> host(bytes);
    hipError_t e = hipGetDevice(&p->device);
    if (e == hipSuccess && bytes) e = limited_malloc(&p->store, bytes);
    if (e == hipSuccess && bytes) {
        size_t at = 0;
        for (size_t i = 0; i < n; ++i) {
            if (lists[i].bytes) memcpy(host.data() + at, lists[i].src, lists[i].bytes);
            *lists[i].dst = (char *)p->store + at;
            at += round256(lists[i].bytes);
        }
        e = hipMemcpy(p->store, host.data(), bytes, hipMemcpyHostToDevice);
    }
    return e;
}

inline bool on_device(const f3s_cross_plan_s *p, hipStream_t stream)
{
    int dev = -1;
    const hipError_t e = stream ? hipStreamGetDevice(stream, &dev) : hipGetDevice(&dev);
    return e == hipSuccess && dev == p->device;
}

// Partial rows of d floats, then their records of `record` floats.
inline size_t parts_bytes(int64_t rows, int32_t d, int32_t record)
{
    return rows ? round256((size_t)rows * d * 4) + round256((size_t)rows * record * 4) : 0;
}

// |scale| log2 e.  Scores that are left out are -inf and stay so under a factor
// that is not 0: a scale of 0 counts as 2^-120, which turns every finite score
// of an f16 or bf16 product below 2^100 into 0 as well.
inline float base2_scale(float scale)
{
    const float s = scale_log2e(scale);
    return s < 0x1p-120f ? 0x1p-120f : s;
}

inline bool workspace_ok(const void *w, size_t have, size_t need)
{
    return need == 0 || (w && aligned(w, 256) && have >= need);
}

inline size_t forward_workspace(const f3s_cross_plan_s *p)
{
    return p ? parts_bytes(p->fwd_parts, p->d, 2) : 0;
}

inline size_t backward_workspace(const f3s_cross_plan_s *p)
{
    if (!p) return 0;
    return round256((size_t)p->q_rows * p->n_heads * 8) + parts_bytes(p->dq_parts, p->d, 0) +
           parts_bytes(p->dkv_parts, 2 * p->d, 0);
}

// A forward call: checked, launched by launch(args, bf16), its pieces joined.
template <typename Launch>
f3s_status_t dense_forward(const f3s_cross_plan_s *p, const void *Q, const void *K, const void *V,
                           f3s_dtype_t dtype, void *O, float *lse, float scale, void *workspace,
                           size_t workspace_bytes, hipStream_t stream, Launch launch)
{
    if (!p || !isfinite(scale)) return set_status(F3S_ERR_INVALID_VALUE);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return set_status(F3S_ERR_UNSUPPORTED);
    if (p->q_rows == 0) return F3S_OK;
    if (!on_device(p, stream)) return set_status(F3S_ERR_INVALID_VALUE);
    if (!Q || !O || !lse || (p->k_rows && (!K || !V)) || !aligned(Q, 16) || !aligned(K, 16) ||
        !aligned(V, 16) || !aligned(O, 16) || !aligned(lse, 4))
        return set_status(F3S_ERR_INVALID_VALUE);
    const size_t need = forward_workspace(p);
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
    FewArgs a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.O = O;
    a.lse = lse;
    a.q = query_rows(p->n_heads, p->g);
    a.n_kv = p->n_kv;
    a.sl2 = base2_scale(scale);
    a.flip = signbit(scale) ? 0x80008000u : 0u;
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + round256((size_t)p->fwd_parts * p->d * 4));
    const bool bf16 = dtype == F3S_DTYPE_BF16;
    hipError_t e = launch(a, bf16);
    if (e == hipSuccess && p->n_fwd_merge) {
        const CrossMergeArgs m = {p->fwd_merge, a.part_o, a.part_ml, O, lse, a.q, 0};
        e = bf16 ? launch_cross_merge_bf16(*p, m, stream)
                 : launch_cross_merge_f16(*p, m, stream);
    }
    return set_status(status_of(e));
}

// A backward call: checked, and launched by launch(args, bf16).
template <typename Launch>
f3s_status_t dense_backward(const f3s_cross_plan_s *p, const void *Q, const void *K, const void *V,
                            f3s_dtype_t dtype, const void *O, const void *dO, const float *lse,
                            void *dQ, void *dK, void *dV, float scale, void *workspace,
                            size_t workspace_bytes, hipStream_t stream, Launch launch)
{
    if (!p || !isfinite(scale)) return set_status(F3S_ERR_INVALID_VALUE);
    if (dtype != F3S_DTYPE_F16 && dtype != F3S_DTYPE_BF16)
        return set_status(F3S_ERR_UNSUPPORTED);
    if (p->q_rows == 0 && p->k_rows == 0) return F3S_OK;
    if (!on_device(p, stream)) return set_status(F3S_ERR_INVALID_VALUE);
    const size_t qb = (size_t)p->q_rows * p->n_heads * p->d * 2;
    const size_t kb = (size_t)p->k_rows * p->n_kv * p->d * 2;
    const size_t lb = (size_t)p->q_rows * p->n_heads * 4;
    const size_t need = backward_workspace(p);
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
    CrossBwdArgs a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.O = O;
    a.G = dO;
    a.lse = lse;
    a.dQ = dQ;
    a.dK = dK;
    a.dV = dV;
    a.q = query_rows(p->n_heads, p->g);
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
    return set_status(status_of(launch(a, dtype == F3S_DTYPE_BF16)));
}

}  // namespace f3s
