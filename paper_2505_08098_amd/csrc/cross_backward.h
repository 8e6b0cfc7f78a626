// Backward of cross attention (instances: cross_backward_f16.hip,
// cross_backward_bf16.hip).  Two passes, neither with atomics:
//
//   k_cross_dq   owns query rows and walks keys: delta = dO . O of its rows
//                (kept beside lse for the other pass), then per tile
//                S^T = K Q^T, dP^T = V dO^T, dS = P (dP - delta),
//                dQ^T += K^T dS^T.
//   k_cross_dkv  owns key rows and walks the query rows of all heads of the
//                group (so that the sum over them needs nothing more):
//                S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
//
// P comes from lse, so nothing of the size of the scores is stored: 7 products
// instead of 5.  As in the forward, the accumulator of the first products is
// the operand of the second in place, each wave has 32 rows of its own side in
// registers, and tiles of 64 rows of the other side pass through LDS for all
// four waves in two buffers.  The matrix units and LDS reads (one operand of
// every product) are the bound.
#pragma once

#include "many_rows.h"

namespace f3s {

struct CrossBwdArgs {
    const void *Q, *K, *V, *O, *G;
    const float *lse;
    float2 *stats;     // per query row and head: lse log2 e, delta
    void *dQ, *dK, *dV;
    float *part_dq;    // [dq_parts][D]
    float *part_dkv;   // [dkv_parts][2 D]: dK, then dV
    QueryRows q;
    int32_t n_kv;
    float sl2;         // |scale| log2 e
    float scale;
    uint32_t flip;     // sign bits: Q is negated in the scores where scale < 0
};

constexpr float kLog2e = 1.4426950408889634f;

// Four columns of a result row from an accumulator.
__device__ __forceinline__ f4 quad(const f16v &x, int k)
{
    return f4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
}

// An O^T-like accumulator's row, scaled and rounded, or as it is into partial sums.
template <int D, int kIn, int D0, int D1>
__device__ __forceinline__ void store_row(const f16v (&x)[(D1 - D0) / 32], float scale, void *to,
                                          int64_t at, float *part, int lane)
{
    const int col = D0 + 4 * (lane >> 5);
#pragma unroll
    for (int d = 0; d < (D1 - D0) / 32; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f4 v = quad(x[d], k);
            if (part)
                *reinterpret_cast<f4 *>(part + 32 * d + 8 * k + col) = v;
            else
                store4<kIn>(to, at * D + 32 * d + 8 * k + col, v * scale);
        }
}

constexpr int dq_waves(int d) { return d <= 64 ? 3 : d <= 128 ? 2 : 1; }
constexpr int dkv_waves(int d) { return d <= 64 ? 2 : 1; }

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dq_waves(D)) void k_cross_dq(CrossBwdArgs a,
                                                                        const DenseItem *items)
{
    using T = ManyTile<D, 32>;
    constexpr int kTile = T::kRows;
    __shared__ __attribute__((aligned(16))) uint8_t s_k[2][T::kBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_v[2][T::kBytes];
    const DenseItem it = items[blockIdx.x];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < it.rows;
    const bool busy = 32 * wave < it.rows;
    const int64_t at = query_row(a.q, it.head, (int64_t)it.row + (there ? mine : 0));

    u4 kr[T::kLoads], vr[T::kLoads];
    const int n = (it.others + kTile - 1) / kTile;
    auto load = [&](int t) {
        T::load(kr, a.K, it.other, a.n_kv, it.head, kTile * t, it.others);
        T::load(vr, a.V, it.other, a.n_kv, it.head, kTile * t, it.others);
    };
    auto store = [&](int t) {
        T::store(s_k[t & 1], kr);
        T::store(s_v[t & 1], vr);
    };
    if (n > 0) load(0);

    h8 q[D / 16], g[D / 16];
    load_rows32<D>(q, a.Q, at, there, a.flip, lane);
    load_rows32<D>(g, a.G, at, there, 0u, lane);
    float delta = 0.f;
    {
        h8 o[D / 16];
        load_rows32<D>(o, a.O, at, there, 0u, lane);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) delta += from16<kIn>(g[c][k]) * from16<kIn>(o[c][k]);
        delta = sum_xor32(delta);
    }
    const float lse2 = there ? a.lse[at] * kLog2e : INFINITY;
    if (there && lane < 32 && it.piece == 0) a.stats[at] = float2{lse2, delta};

    f16v dq[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) dq[d] = zero16();
    if (n > 0) {
        store(0);
        load(n > 1 ? 1 : 0);
    }
    for (int t = 0; t < n; ++t) {
        __syncthreads();
        if (t + 1 < n) {
            store(t + 1);
            load(min(t + 2, n - 1));
        }
        if (!busy) continue;
        const uint8_t *k = s_k[t & 1], *v = s_v[t & 1];
        const int left = it.others - kTile * t;
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            f16v s = zero16(), dp = zero16();
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                s = mfma32<kIn>(T::rows32(k, 32 * b, c, lane), q[c], s);
                dp = mfma32<kIn>(T::rows32(v, 32 * b, c, lane), g[c], dp);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.sl2, -lse2)) * (dp[e] - delta);
            if (left < kTile) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * b + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3) >= left) s[e] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const h8 ds = pack8<kIn>(s, c);
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
                    dq[d] = mfma32<kIn>(T::cols32(k, 32 * b + 16 * c, 32 * d, lane), ds, dq[d]);
            }
        }
    }
    if (there)
        store_row<D, kIn, 0, D>(dq, a.scale, a.dQ, at,
                          it.part >= 0 ? a.part_dq + ((int64_t)it.part + mine) * D : nullptr,
                          lane);
}

template <int D>
struct DkvTiles {
    using T = ManyTile<D, 32>;
    __attribute__((aligned(16))) uint8_t q[2][T::kBytes], g[2][T::kBytes];
    __attribute__((aligned(16))) float lse[2][T::kRows], delta[2][T::kRows];
};

// Columns D0 .. D1 - 1 of dK and dV (all of them up to d = 128; wider rows take
// two workgroups, each with half of the sums in its registers).
template <int D, int kIn, int D0, int D1>
__device__ __forceinline__ void cross_dkv(const CrossBwdArgs &a, const DenseItem &it,
                                          DkvTiles<D> &s)
{
    using T = ManyTile<D, 32>;
    constexpr int kTile = T::kRows;
    auto &s_q = s.q, &s_g = s.g;
    auto &s_lse = s.lse, &s_delta = s.delta;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < it.rows;
    const bool busy = 32 * wave < it.rows;
    const int64_t at = ((int64_t)it.row + (there ? mine : 0)) * a.n_kv + it.head;

    u4 qr[T::kLoads], gr[T::kLoads];
    float2 sr = {0.f, 0.f};
    const int n = (it.others + kTile - 1) / kTile;
    auto load = [&](int t) {
#pragma unroll
        for (int j = 0; j < T::kLoads; ++j) {
            const int f = (int)threadIdx.x + kManyThreads * j, row = T::row_of(j);
            const int64_t r = query_row(
                a.q, it.head, (int64_t)it.other + min(kTile * t + row, it.others - 1));
            const int64_t byte = r * (2 * D) + (f - row * T::kPieces) * 16;
            qr[j] = *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(a.Q) + byte);
            gr[j] = *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(a.G) + byte);
        }
        if (threadIdx.x < kTile) {
            const int row = kTile * t + (int)threadIdx.x;
            sr = a.stats[query_row(a.q, it.head, (int64_t)it.other + min(row, it.others - 1))];
            if (row >= it.others) sr.x = INFINITY;  // (P = 0)
        }
    };
    auto store = [&](int t) {
        T::store(s_q[t & 1], qr);
        T::store(s_g[t & 1], gr);
        if (threadIdx.x < kTile) {
            s_lse[t & 1][threadIdx.x] = sr.x;
            s_delta[t & 1][threadIdx.x] = sr.y;
        }
    };
    if (n > 0) load(0);
    h8 k[D / 16], v[D / 16];
    load_rows32<D>(k, a.K, at, there, a.flip, lane);  // (the sign on the rows that stay)
    load_rows32<D>(v, a.V, at, there, 0u, lane);
    constexpr int kCols = (D1 - D0) / 32;
    f16v dk[kCols], dv[kCols];
#pragma unroll
    for (int d = 0; d < kCols; ++d) dk[d] = dv[d] = zero16();
    if (n > 0) {
        store(0);
        load(n > 1 ? 1 : 0);
    }
    for (int t = 0; t < n; ++t) {
        __syncthreads();
        if (t + 1 < n) {
            store(t + 1);
            load(min(t + 2, n - 1));
        }
        if (!busy) continue;
        const uint8_t *q = s_q[t & 1], *g = s_g[t & 1];
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            f16v s = zero16(), dp = zero16();
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                s = mfma32<kIn>(T::rows32(q, 32 * b, c, lane), k[c], s);
                dp = mfma32<kIn>(T::rows32(g, 32 * b, c, lane), v[c], dp);
            }
            f16v p;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 32 * b + 8 * r + 4 * (lane >> 5);
                const f4 l = *reinterpret_cast<const f4 *>(&s_lse[t & 1][row]);
                const f4 w = *reinterpret_cast<const f4 *>(&s_delta[t & 1][row]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x =
                        __builtin_amdgcn_exp2f(fmaf(s[4 * r + e], a.sl2, -l[e]));
                    p[4 * r + e] = x;
                    s[4 * r + e] = x * (dp[4 * r + e] - w[e]);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const h8 pp = pack8<kIn>(p, c), ds = pack8<kIn>(s, c);
#pragma unroll
                for (int d = 0; d < kCols; ++d) {
                    const int row = 32 * b + 16 * c, col = D0 + 32 * d;
                    dv[d] = mfma32<kIn>(T::cols32(g, row, col, lane), pp, dv[d]);
                    dk[d] = mfma32<kIn>(T::cols32(q, row, col, lane), ds, dk[d]);
                }
            }
        }
    }
    if (!there) return;
    float *part = it.part >= 0 ? a.part_dkv + ((int64_t)it.part + mine) * (2 * D) : nullptr;
    store_row<D, kIn, D0, D1>(dk, a.scale, a.dK, at, part, lane);
    store_row<D, kIn, D0, D1>(dv, 1.f, a.dV, at, part ? part + D : nullptr, lane);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dkv_waves(D)) void k_cross_dkv(
    CrossBwdArgs a, const DenseItem *items)
{
    __shared__ DkvTiles<D> tiles;
    if constexpr (D <= 128) {
        cross_dkv<D, kIn, 0, D>(a, items[blockIdx.x], tiles);
    } else {
        constexpr int kHalf = (D / 2 + 31) / 32 * 32;
        if (blockIdx.x & 1)
            cross_dkv<D, kIn, kHalf, D>(a, items[blockIdx.x >> 1], tiles);
        else
            cross_dkv<D, kIn, 0, kHalf>(a, items[blockIdx.x >> 1], tiles);
    }
}

// Rows of split ranges: their partial sums added in order, D / 4 threads to a
// row.  kKeys: dK and dV, else dQ.
template <int D, int kIn, bool kKeys>
__global__ __launch_bounds__(256) void k_cross_sum(CrossBwdArgs a, const DenseMerge *merges,
                                                   int blocks)
{
    constexpr int kWidth = kKeys ? 2 * D : D, kPer = 256 / (D / 4), kAhead = 8;
    const int rec = (int)blockIdx.x / blocks;
    const DenseMerge g = merges[rec];
    const int r = ((int)blockIdx.x - rec * blocks) * kPer + (int)threadIdx.x / (D / 4);
    const int c = threadIdx.x % (D / 4) * 4;
    if (threadIdx.x >= kPer * (D / 4) || r >= g.rows) return;
    const float *part = kKeys ? a.part_dkv : a.part_dq;
    const int64_t at = kKeys ? ((int64_t)g.row + r) * a.n_kv + g.head
                             : query_row(a.q, g.head, (int64_t)g.row + r);
#pragma unroll
    for (int w = 0; w < kWidth / D; ++w) {
        f4 sum = f4{0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < g.count; p += kAhead) {
            f4 x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                x[k] = *reinterpret_cast<const f4 *>(
                    part + ((int64_t)g.part + r + (int64_t)g.stride * min(p + k, g.count - 1)) *
                               kWidth + w * D + c);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (p + k < g.count) sum += x[k];
        }
        store4<kIn>(!kKeys ? a.dQ : w ? a.dV : a.dK, at * D + c, sum * (w ? 1.f : a.scale));
    }
}

template <int D, int kIn>
hipError_t launch_cross_backward_d(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                   hipStream_t s)
{
    constexpr int kPer = 256 / (D / 4);
    if (p.n_dq) k_cross_dq<D, kIn><<<p.n_dq, kManyThreads, 0, s>>>(a, p.dq);
    if (p.n_dkv)
        k_cross_dkv<D, kIn><<<(unsigned)(D <= 128 ? p.n_dkv : 2 * p.n_dkv), kManyThreads, 0, s>>>(
            a, p.dkv);
    if (p.n_dq_merge) {
        const int blocks = (p.dq_merge_rows + kPer - 1) / kPer;
        k_cross_sum<D, kIn, false><<<(unsigned)(p.n_dq_merge * blocks), 256, 0, s>>>(
            a, p.dq_merge, blocks);
    }
    if (p.n_dkv_merge) {
        const int blocks = (p.dkv_merge_rows + kPer - 1) / kPer;
        k_cross_sum<D, kIn, true><<<(unsigned)(p.n_dkv_merge * blocks), 256, 0, s>>>(
            a, p.dkv_merge, blocks);
    }
    return hipGetLastError();
}

hipError_t launch_cross_backward_f16(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                     hipStream_t s);
hipError_t launch_cross_backward_bf16(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                      hipStream_t s);

}  // namespace f3s
