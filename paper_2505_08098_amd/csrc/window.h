// Causal self-attention in which a token sees the newest `window` tokens and the first
// `sinks` ones (f3s_window_forward, f3s_window_backward): the kernels of cross attention
// (many_rows.h, cross_backward.h) over the keys that a tile's rows see.
//
// A tile of 128 query rows (128 / g tokens of a key head) walks the sinks, then the keys
// from its first token's window to its last token (WindowKeys): what it reads beside the
// window is the sinks' tile and its own length.  A wave of 32 rows leaves out tiles that
// none of its rows sees and masks, score by score, only those that some do not see (the
// window's edge and the diagonal).  In the pass of dK and dV a tile of 128 keys walks the
// query rows from its first key on to the end of its last key's window; the sinks, which
// all later rows see, are tiles of their own.
//
// 32,749 tokens, 32 heads of 128 over 8, bf16, window 4,096: 2,010 to 2,120 us by card, 970
// to 1,030 TFLOP/s (the bound is many_rows.h's).  Training on two sequences of 8,100, 16 heads
// of 128 over 4, window 1,024, 16 sinks: 690 to 714 us, under the profiler 162 forward, 222 dQ,
// 331 dK and dV, 7.5 sums.  16 of 300 to 1,025 tokens padded, 12 heads of 64, causal: 117 to
// 124 us in all (31, 43 and 54).
//
// A few newest query rows leave three waves of four without any, which costs little, since
// bytes count: one token over 8,192 keys of 64 sequences, 32 heads of 128 over 8, 352 us in
// graphs (6.1 TB/s), 366 by the kernel of 16 rows (few_rows.h, as cross attention); of one
// sequence, where its launch and chain count, 12.0 and 8.7.
#pragma once

#include "cross_backward.h"

namespace f3s {

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, many_waves(D)) void k_window(
    FewArgs a, const WindowItem *items, WindowRule rule)
{
    const WindowItem it = items[blockIdx.x];
    many_rows<D, kIn>(a, it, rule);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dq_waves(D)) void k_window_dq(
    CrossBwdArgs a, const WindowItem *items, WindowRule rule)
{
    const WindowItem it = items[blockIdx.x];
    dense_dq<D, kIn>(a, it, rule);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dkv_waves(D)) void k_window_dkv(
    CrossBwdArgs a, const WindowItem *items, WindowRule rule)
{
    __shared__ DkvBuffer<D> s0, s1;
    __shared__ __attribute__((aligned(16)))
    uint8_t s_v[dkv_v_in_lds(D) ? ManyTile<D, kManyRows>::kBytes : 16];
    const WindowItem it = items[blockIdx.x / dkv_halves(D)];
    if constexpr (dkv_halves(D) == 1) {
        dense_dkv<D, kIn, 0, D>(a, it, rule, s0, s1, s_v);
    } else {
        constexpr int kHalf = (D / 2 + 31) / 32 * 32;
        if (blockIdx.x & 1)
            dense_dkv<D, kIn, kHalf, D>(a, it, rule, s0, s1, s_v);
        else
            dense_dkv<D, kIn, 0, kHalf>(a, it, rule, s0, s1, s_v);
    }
}

template <int D, int kIn>
hipError_t launch_window_d(const f3s_window_plan_s &p, const FewArgs &a, hipStream_t s)
{
    if (p.n_fwd)
        k_window<D, kIn><<<p.n_fwd, kManyThreads, 0, s>>>(
            a, p.window_fwd, p.rule);
    return hipGetLastError();
}

template <int D, int kIn>
hipError_t launch_window_backward_d(const f3s_window_plan_s &p, const CrossBwdArgs &a,
                                    hipStream_t s)
{
    if (p.n_dq) k_window_dq<D, kIn><<<p.n_dq, kManyThreads, 0, s>>>(a, p.window_dq, p.rule);
    if (p.n_dkv)
        k_window_dkv<D, kIn><<<(unsigned)(p.n_dkv * dkv_halves(D)), kManyThreads, 0, s>>>(
            a, p.window_dkv, p.rule);
    return launch_cross_sums_d<D, kIn>(p, a, s);
}

hipError_t launch_window_f16(const f3s_window_plan_s &p, const FewArgs &a, hipStream_t s);
hipError_t launch_window_bf16(const f3s_window_plan_s &p, const FewArgs &a, hipStream_t s);
hipError_t launch_window_backward_f16(const f3s_window_plan_s &p, const CrossBwdArgs &a,
                                      hipStream_t s);
hipError_t launch_window_backward_bf16(const f3s_window_plan_s &p, const CrossBwdArgs &a,
                                       hipStream_t s);

}  // namespace f3s
