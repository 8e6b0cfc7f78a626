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
// registers, and tiles of 32 rows of the other side (d = 32: 64) pass through LDS
// for all four waves in two buffers.  As in the forward power is the bound, and in
// k_cross_dkv LDS reads (one operand of every product, and V): 2 x 4,050 x 4,050, 16
// heads of 128 over 4, bf16, takes 413 us for dQ and 558 for dK and dV, 970 TFLOP/s of the
// 7 products.
//
// P and dS enter the second products in the inputs' type, as P does in the forward,
// and for its reasons; delta comes from the rounded O, since the exact one would take
// two more products, a sweep ahead of dQ's.
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

// Rows of a tile of the other side (64 for short rows: 4 KB to fill at once).
constexpr int bwd_tile(int d) { return d <= 32 ? 64 : 32; }
constexpr float kLog2e = 1.4426950408889634f;

constexpr int dq_waves(int d) { return d <= 32 ? 4 : d <= 64 ? 3 : d <= 128 ? 2 : 1; }
constexpr int dkv_halves(int d) { return d <= 128 ? 1 : 2; }
constexpr int dkv_waves(int d) { return d <= 64 ? 3 : d <= 128 ? 2 : 1; }

template <int D, int kIn, typename Item>
__device__ __forceinline__ void dense_dq(const CrossBwdArgs &a, const Item &it,
                                         const WindowRule &rule)
{
    constexpr bool kWindow = std::is_same<Item, WindowItem>::value;
    using T = ManyTile<D, bwd_tile(D)>;
    constexpr int kTile = T::kRows;
    __shared__ __attribute__((aligned(16))) uint8_t s_k0[T::kBytes], s_k1[T::kBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_v0[T::kBytes], s_v1[T::kBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < it.rows;
    const bool busy = 32 * wave < it.rows;
    const RowPositions at_p = row_positions(a.q, it, wave, there ? mine : 0);
    const int64_t at = query_row(a.q, it.head, (int64_t)it.row + (there ? mine : 0));

    T tk, tv;
    const uint32_t row_bytes = (uint32_t)a.n_kv * (2 * D);
    const uint64_t base = (uint64_t)key_base(it) * row_bytes + (uint32_t)it.head * (2 * D);
    const uint8_t *const K = reinterpret_cast<const uint8_t *>(a.K) + base;
    const uint8_t *const V = reinterpret_cast<const uint8_t *>(a.V) + base;
    auto fetch = [&](int t, auto buf) {
        const KeyRun run = key_run(it, kTile * t);
        const int first = run.key, last = kWindow ? max(run.left - 1, 0) : run.left - 1;
        const uint64_t at = (uint64_t)first * row_bytes;
        // (behind the range: the last row again)
        auto offset = [&](int row) { return (uint32_t)min(row, last) * row_bytes; };
        tk.fetch(buf.kIndex ? s_k1 : s_k0, K + at, offset);
        tv.fetch(buf.kIndex ? s_v1 : s_v0, V + at, offset);
    };
    auto put = [&](int, auto buf) {
        tk.put(buf.kIndex ? s_k1 : s_k0);
        tv.put(buf.kIndex ? s_v1 : s_v0);
    };

    h8 q[D / 16], g[D / 16];
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
    load_rows32<D>(q, a.Q, at, there, a.flip, lane);
    float lse2 = there ? a.lse[at] * kLog2e : INFINITY;
    if (kWindow && lse2 == -INFINITY) lse2 = INFINITY;  // (it sees nothing: P = 0)
    if (there && lane < 32 && it.piece == 0) a.stats[at] = float2{lse2, delta};

    f16v dq[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) dq[d] = zero16();
    auto work = [&](int t, auto buf) {
        if (!busy) return;
        const uint8_t *k = buf.kIndex ? s_k1 : s_k0, *v = buf.kIndex ? s_v1 : s_v0;
        const KeyRun run = key_run(it, kTile * t);
        const int left = run.left;
        if (kWindow &&
            (left <= 0 || window_none(rule, at_p.first, at_p.last, run.key, min(left, kTile))))
            return;
        const bool some = kWindow && (left < kTile || !window_all(rule, at_p.first, at_p.last,
                                                                  run.key, kTile));
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            if (kTile > 32) __builtin_amdgcn_sched_barrier(0);  // (one block at a time)
            f16v s = zero16(), dp = zero16();
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                s = mfma32<kIn>(T::rows32(k, 32 * b, c, lane), q[c], s);
                dp = mfma32<kIn>(T::rows32(v, 32 * b, c, lane), g[c], dp);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.sl2, -lse2)) * (dp[e] - delta);
            if constexpr (kWindow) {
                if (some) {
                    const uint32_t bits =
                        lane_bits(window_bits(rule, at_p.mine, run.key + 32 * b) &
                                      bits_to(left - 32 * b - 1),
                                  lane);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = kept_value(s[e], bits, e);
                }
            } else if (left < kTile) {
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
        products_done();
    };
    walk_tiles<T::kDirect>((it.others + kTile - 1) / kTile, fetch, put, work);
    uint8_t *const lds = wave == 0 ? s_k0 : wave == 1 ? s_k1 : wave == 2 ? s_v0 : s_v1;
    const int rows = it.rows - 32 * wave;
    __syncthreads();  // nobody reads the tiles
    if (it.part >= 0)
        store_part32<D, T::kBytes / 128 / 32 * 32>(
            lds, dq, 1.f, a.part_dq + ((int64_t)it.part + 32 * wave) * D, D, rows, lane);
    else
        store_rows32<D, kIn, D>(
            lds, dq, a.scale, a.dQ,
            [&](int r) { return query_row(a.q, it.head, (int64_t)it.row + 32 * wave + r); }, rows,
            0, lane);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dq_waves(D)) void k_cross_dq(CrossBwdArgs a,
                                                                        const DenseItem *items)
{
    const DenseItem it = items[blockIdx.x];
    dense_dq<D, kIn>(a, it, {});
}

// d = 64 to 128: the sums of dK and dV leave no room for both K and V beside
// them if two waves (three of d = 64) are to share a SIMD, which is worth more
// (d = 128, 16 heads over 4, 2 x 4,050 x 4,050: 1,007 us against 1,424 with one
// wave, the rest of the kernel as it then was); V's rows stay in LDS.
constexpr bool dkv_v_in_lds(int d) { return d > 32 && d <= 128; }

template <int D>
using DkvTile = ManyTile<D, bwd_tile(D)>;

// P enters dV's product times 2^12 in f16, whose least normal number is 2^-14: a
// row's probabilities sum to 1, so those of a few ten thousand keys would lose bits
// (1.3% of each at a million keys, the same way for all), and no scaling of dO helps,
// since P has none of it.  They keep 11 bits down to 2^-26, and 2^12 leaves 16 times
// of room above 1 for what lse is off by.  The factor costs nothing: it is added to
// the exponent with lse, dS takes it out within the subtraction of delta (exactly),
// and dV as it is stored.  bf16 has fp32's exponents.
template <int kIn>
constexpr float kPUp = kIn == kInF16 ? 0x1p12f : 1.f;
template <int kIn>
constexpr float kPUpLog2 = kIn == kInF16 ? 12.f : 0.f;

// A tile of query rows and what belongs to it.
template <int D>
struct DkvBuffer {
    __attribute__((aligned(16))) uint8_t q[DkvTile<D>::kBytes], g[DkvTile<D>::kBytes];
    __attribute__((aligned(16))) float lse[DkvTile<D>::kRows], delta[DkvTile<D>::kRows];
};

// Columns D0 .. D1 - 1 of dK and dV (all of them up to d = 128; wider rows take
// two workgroups, each with half of the sums in its registers).
template <int D, int kIn, int D0, int D1, typename Item>
__device__ __forceinline__ void dense_dkv(const CrossBwdArgs &a, const Item &it,
                                          const WindowRule &rule, DkvBuffer<D> &s0,
                                          DkvBuffer<D> &s1, uint8_t *s_v)
{
    constexpr bool kWindow = std::is_same<Item, WindowItem>::value;
    using T = DkvTile<D>;
    using TV = ManyTile<D, kManyRows>;
    constexpr bool kVInLds = dkv_v_in_lds(D);
    constexpr int kTile = T::kRows, kWidth = D1 - D0;
    constexpr float kPDown = 1.f / kPUp<kIn>;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < it.rows;
    const bool busy = 32 * wave < it.rows;
    const int64_t at = ((int64_t)it.row + (there ? mine : 0)) * a.n_kv + it.head;

    T tq, tg;
    float2 sr = {0.f, 0.f};
    auto fetch = [&](int t, auto buf) {
        // offsets from the first row's token on
        const uint32_t first = (uint32_t)it.other + kTile * t;
        const int last = it.others - 1 - kTile * t;  // (behind it: the last row again)
        const uint32_t token = row_token(a.q, first);
        auto offset = [&](int row) {
            const uint32_t r = first + (uint32_t)min(row, last), k = row_token(a.q, r) - token;
            return r - token * (uint32_t)a.q.g + k * (uint32_t)(a.q.n_heads - a.q.g);
        };
        const uint64_t at = (uint64_t)token * a.q.n_heads + (uint32_t)(it.head * a.q.g);
        auto bytes = [&](int row) { return offset(row) * (2 * D); };
        auto &to = buf.kIndex ? s1 : s0;
        tq.fetch(to.q, reinterpret_cast<const uint8_t *>(a.Q) + at * (2 * D), bytes);
        tg.fetch(to.g, reinterpret_cast<const uint8_t *>(a.G) + at * (2 * D), bytes);
        // (by all threads: a load in a branch would be waited for at its end)
        sr = a.stats[at + offset((int)threadIdx.x % kTile)];
    };
    auto put = [&](int t, auto buf) {
        auto &to = buf.kIndex ? s1 : s0;
        tq.put(to.q);
        tg.put(to.g);
        if (threadIdx.x < kTile) {
            to.lse[threadIdx.x] =
                kTile * t + (int)threadIdx.x < it.others ? sr.x - kPUpLog2<kIn>
                                                         : INFINITY;  // (P = 0)
            to.delta[threadIdx.x] = sr.y * kPDown;
        }
    };
    h8 k[D / 16], v[kVInLds ? 1 : D / 16];
    load_rows32<D>(k, a.K, at, there, a.flip, lane);  // (the sign on the rows that stay)
    if constexpr (kVInLds) {
        for (int f = threadIdx.x; f < kManyRows * TV::kPieces; f += kManyThreads) {
            const int row = f / TV::kPieces, piece = f % TV::kPieces;
            const int64_t r = ((int64_t)it.row + min(row, it.rows - 1)) * a.n_kv + it.head;
            *reinterpret_cast<u4 *>(s_v + row * TV::kStride +
                                    (piece ^ TV::swizzle(row & 31)) * 16) =
                *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(a.V) +
                                              r * (2 * D) + piece * 16);
        }
    } else {
        load_rows32<D>(v, a.V, at, there, 0u, lane);
    }
    constexpr int kCols = kWidth / 32;
    f16v dk[kCols], dv[kCols];
#pragma unroll
    for (int d = 0; d < kCols; ++d) dk[d] = dv[d] = zero16();
    auto work = [&](int t, auto buf) {
        if (!busy) return;
        const auto &from = buf.kIndex ? s1 : s0;
        const uint8_t *q = from.q, *g = from.g;
        bool some = false;  // some query rows do not see some keys
        int key = 0;        // the wave's first
        if constexpr (kWindow) {
            const int first = it.other + kTile * t;
            const int last = it.other + min(kTile * (t + 1), it.others) - 1;
            const int p0 = (int)row_token(a.q, first) + it.shift;
            const int p1 = (int)row_token(a.q, last) + it.shift;
            const int key0 = it.row - it.key0 + 32 * wave, n = min(32, it.rows - 32 * wave);
            if (window_none(rule, p0, p1, key0, n)) return;
            some = !window_all(rule, p0, p1, key0, n);
            key = key0;
        }
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            if (kTile > 32) __builtin_amdgcn_sched_barrier(0);  // (one block at a time)
            f16v x = zero16(), dp = zero16();
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                x = mfma32<kIn>(T::rows32(q, 32 * b, c, lane), k[c], x);
                dp = mfma32<kIn>(T::rows32(g, 32 * b, c, lane),
                                 kVInLds ? TV::rows32(s_v, 32 * wave, c, lane) : v[c], dp);
            }
            if constexpr (kWindow) {
                if (some) {
                    // The rows that see a key stand one behind the other: from the first of
                    // the token at its position on to the last of its window's last token,
                    // or, for a sink, without end.
                    int l = lane;
                    // (d = 64 and 128 have no register left that would hold it until here)
                    if constexpr (D == 64 || D == 128) asm volatile("" : "+v"(l));
                    const int j = key + (l & 31);
                    auto row = [&](int64_t r) { return (int)max(min(r, (int64_t)64), (int64_t)0); };
                    const int64_t from =
                        (int64_t)(j - it.shift) * a.q.g - (it.other + kTile * t + 32 * b);
                    const int64_t to =
                        j < rule.sinks ? 64 : from + (int64_t)rule.window * a.q.g;
                    const uint32_t bits =
                        lane_bits(bits_to(row(to) - 1) & ~bits_to(row(from) - 1), l);
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = kept_score(x[e], bits, e);
                }
            }
            f16v p;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 32 * b + 8 * r + 4 * (lane >> 5);
                const f4 l = *reinterpret_cast<const f4 *>(&from.lse[row]);
                const f4 w = *reinterpret_cast<const f4 *>(&from.delta[row]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y =
                        __builtin_amdgcn_exp2f(fmaf(x[4 * r + e], a.sl2, -l[e]));
                    p[4 * r + e] = y;
                    x[4 * r + e] = y * fmaf(dp[4 * r + e], kPDown, -w[e]);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const h8 pp = pack8<kIn>(p, c), ds = pack8<kIn>(x, c);
#pragma unroll
                for (int d = 0; d < kCols; ++d) {
                    const int row = 32 * b + 16 * c, col = D0 + 32 * d;
                    dv[d] = mfma32<kIn>(T::cols32(g, row, col, lane), pp, dv[d]);
                    dk[d] = mfma32<kIn>(T::cols32(q, row, col, lane), ds, dk[d]);
                }
            }
        }
        products_done();
    };
    walk_tiles<T::kDirect>((it.others + kTile - 1) / kTile, fetch, put, work);
    // (two waves to a buffer)
    constexpr int kOwn = sizeof(DkvBuffer<D>) / 2 / 16 * 16, kChunk = kOwn / 128 / 32 * 32;
    static_assert(kOwn >= 64 * kWidth && kChunk >= 32, "room for a wave's rows");
    uint8_t *const lds = reinterpret_cast<uint8_t *>(wave & 2 ? &s1 : &s0) + (wave & 1) * kOwn;
    const int rows = it.rows - 32 * wave;
    __syncthreads();  // nobody reads the tiles
    if (it.part >= 0) {
        float *part = a.part_dkv + ((int64_t)it.part + 32 * wave) * (2 * D) + D0;
        store_part32<kWidth, kChunk>(lds, dk, 1.f, part, 2 * D, rows, lane);
        store_part32<kWidth, kChunk>(lds, dv, kPDown, part + D, 2 * D, rows, lane);
        return;
    }
    auto row = [&](int r) { return ((int64_t)it.row + 32 * wave + r) * a.n_kv + it.head; };
    store_rows32<D, kIn, kWidth>(lds, dk, a.scale, a.dK, row, rows, D0, lane);
    store_rows32<D, kIn, kWidth>(lds, dv, kPDown, a.dV, row, rows, D0, lane);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, dkv_waves(D)) void k_cross_dkv(
    CrossBwdArgs a, const DenseItem *items)
{
    __shared__ DkvBuffer<D> s0, s1;
    __shared__ __attribute__((aligned(16)))
    uint8_t s_v[dkv_v_in_lds(D) ? ManyTile<D, kManyRows>::kBytes : 16];
    const DenseItem it = items[blockIdx.x / dkv_halves(D)];
    if constexpr (dkv_halves(D) == 1) {
        dense_dkv<D, kIn, 0, D>(a, it, {}, s0, s1, s_v);
    } else {
        constexpr int kHalf = (D / 2 + 31) / 32 * 32;
        if (blockIdx.x & 1)
            dense_dkv<D, kIn, kHalf, D>(a, it, {}, s0, s1, s_v);
        else
            dense_dkv<D, kIn, 0, kHalf>(a, it, {}, s0, s1, s_v);
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

// The partial sums of a plan's dQ and of its dK and dV.
template <int D, int kIn>
hipError_t launch_cross_sums_d(const f3s_cross_plan_s &p, const CrossBwdArgs &a, hipStream_t s)
{
    constexpr int kPer = 256 / (D / 4);
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

template <int D, int kIn>
hipError_t launch_cross_backward_d(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                   hipStream_t s)
{
    if (p.n_dq) k_cross_dq<D, kIn><<<p.n_dq, kManyThreads, 0, s>>>(a, p.dq);
    if (p.n_dkv)
        k_cross_dkv<D, kIn><<<(unsigned)(p.n_dkv * dkv_halves(D)), kManyThreads, 0, s>>>(
            a, p.dkv);
    return launch_cross_sums_d<D, kIn>(p, a, s);
}

hipError_t launch_cross_backward_f16(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                     hipStream_t s);
hipError_t launch_cross_backward_bf16(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                      hipStream_t s);

}  // namespace f3s
