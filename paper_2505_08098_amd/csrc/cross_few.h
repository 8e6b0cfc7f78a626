// Forward of cross attention for few query rows (single tokens), and the
// joining of partial results (instances: cross_few_f16.hip, cross_few_bf16.hip).
#pragma once

#include "few_rows.h"

namespace f3s {

struct CrossMergeArgs {
    const DenseMerge *merges;
    const float *part_o, *part_ml;
    void *O;
    float *lse;
    QueryRows q;
    int32_t blocks;  // workgroups per record
};

template <int D, int kIn>
__global__ __launch_bounds__(64 * kFewWaves, few_waves(D, false)) void k_cross_few(
    FewArgs a, const DenseItem *items)
{
    const DenseItem d = items[blockIdx.x];
    FewItem it = {};
    it.row = d.row;
    it.rows = d.rows;
    it.head = d.head;
    it.key = d.other;
    it.begin = 0;
    it.end = d.others;
    it.causal = false;
    it.part = d.part;
    few_rows<D, kIn, false>(a, it);
}

// Rows of split ranges from their partial results.
template <int D, int kIn, bool kSplit>
__global__ __launch_bounds__(256) void k_cross_join(CrossMergeArgs a)
{
    constexpr int kPer = kSplit ? 1 : 256 / (D / 4);
    const int rec = (int)blockIdx.x / a.blocks;
    const DenseMerge g = a.merges[rec];
    const int r = ((int)blockIdx.x - rec * a.blocks) * kPer +
                  (kSplit ? 0 : (int)threadIdx.x / (D / 4));
    if (r >= g.rows || (!kSplit && (int)threadIdx.x >= kPer * (D / 4))) return;
    join_row<D, kIn, kIn, kSplit>(a.part_o, a.part_ml, {(int64_t)g.part + r, g.stride, g.count},
                             {0, 0, 0}, query_row(a.q, g.head, (int64_t)g.row + r), a.O, a.lse);
}

template <int D, int kIn>
hipError_t launch_cross_few_d(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s)
{
    if (p.n_fwd) k_cross_few<D, kIn><<<p.n_fwd, 64 * kFewWaves, 0, s>>>(a, p.fwd);
    return hipGetLastError();
}

template <int D, int kIn>
hipError_t launch_cross_merge_d(const f3s_cross_plan_s &p, CrossMergeArgs a, hipStream_t s)
{
    constexpr int kPer = 256 / (D / 4);
    if (!p.n_fwd_merge) return hipSuccess;
    const bool split = (int64_t)p.n_fwd_merge * p.fwd_merge_rows <= kSplitJoins;
    a.blocks = split ? p.fwd_merge_rows : (p.fwd_merge_rows + kPer - 1) / kPer;
    const unsigned grid = (unsigned)(p.n_fwd_merge * a.blocks);
    if (split)
        k_cross_join<D, kIn, true><<<grid, 256, 0, s>>>(a);
    else
        k_cross_join<D, kIn, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

#define F3S_FOR_D(d, call)                \
    switch (d) {                          \
    case 32: return call(32);             \
    case 64: return call(64);             \
    case 96: return call(96);             \
    case 128: return call(128);           \
    case 160: return call(160);           \
    case 192: return call(192);           \
    case 224: return call(224);           \
    default: return call(256);            \
    }

hipError_t launch_cross_few_f16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s);
hipError_t launch_cross_few_bf16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s);
hipError_t launch_cross_merge_f16(const f3s_cross_plan_s &p, const CrossMergeArgs &a,
                                  hipStream_t s);
hipError_t launch_cross_merge_bf16(const f3s_cross_plan_s &p, const CrossMergeArgs &a,
                                   hipStream_t s);

}  // namespace f3s
