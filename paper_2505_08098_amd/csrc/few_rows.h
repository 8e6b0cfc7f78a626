// Attention of at most 16 query rows to a range of keys: the kernel of single
// tokens (f3s_cache_attend over the 8-bit cache, f3s_cross_forward over 16-bit
// K and V).
//
// With so few rows every byte of K and V is used for a handful of products, so
// the pass is bound by reading them.  The four waves of a workgroup take the
// range's tiles of 32 keys in turn, each with a running maximum, sum and
// output of its own, and meet once, at the end; the loads of a wave's next
// tile are under way while it works on the last.
//
// Per tile:  S^T = K Q^T (a lane holds one query row and 8 keys), the softmax
// in base 2 against the running maximum, O^T += V^T P^T.  K and V pass through
// the wave's own part of LDS, loaded in whole 16-byte pieces of consecutive
// rows and read back as matrix operands (V transposed).
//
// Cached keys and values stay codes until they are operands: every code is
// exact in f16 and bf16, the power of two of a key multiplies its score, and
// that of a value its probability, taken relative to the largest power that the
// row has seen so far (both exactly), so that P V runs in f16 with 11 bits of P
// whatever the values' size.
//
// One token of 64 sequences of 1,500 to 4,097 keys, 8 key heads of 128 in bf16: 135
// us, 5.5 TB/s; of 500 to 8,192 cached keys: 116 us, 4.9 TB/s (a copy of 2 GiB
// moves 4.8).
//
// Over 16-bit K and V the probabilities are rounded to the inputs' type, as in
// many_rows.h: a bf16 result is off by 0.0021 of its size instead of 0.0017.
#pragma once

#include "dense_common.h"

namespace f3s {

constexpr int kFewRows = 16;
constexpr int kFewKeys = 32;
constexpr int kFewWaves = 4;

// Waves per SIMD, as many as the registers hold without spills: loads of more
// waves are in flight.
constexpr int few_waves(int d, bool cache)
{
    return cache ? (d <= 64 ? 4 : d <= 160 ? 3 : 2)
                 : (d <= 32 ? 4 : d <= 64 ? 3 : d <= 128 ? 2 : 1);
}

// What a workgroup does.
struct FewItem {
    int64_t row;         // first query row of the key head
    int32_t rows;        // 1..16
    int32_t head;        // key head
    int64_t key;         // 16-bit K, V: row of the range's key 0; cache: unused
    const int32_t *table;  // cache: the pages of position 0, 1, ...
    int32_t table_len;
    int32_t begin, end;  // keys (positions), begin a multiple of 32 in the cache
    int32_t limit;       // keys that the first token's rows see (causal), or end
    int32_t first;       // rows of the first token before `row` (row's index in its sequence)
    bool causal;         // each next token sees one key more
    int64_t part;        // first partial row, -1: final
};

struct FewArgs {
    const void *Q, *K, *V;
    void *O;
    float *lse;
    float *part_o;   // [partial rows][D]
    float *part_ml;  // [partial rows][2]
    QueryRows q;
    int32_t n_kv;
    float sl2;       // |scale| log2 e
    uint32_t flip;   // sign bits: Q is negated where scale < 0
    // cache
    const uint8_t *k, *v, *k_exp, *v_exp;
    int32_t n_pages, page_shift;
};

template <int D, bool kCache>
struct FewTile {
    static constexpr int kRowBytes = kCache ? D : 2 * D;
    static constexpr int kPieces = kRowBytes / 16;              // 16-byte pieces of a row
    static constexpr int kLoads = kFewKeys * kPieces / 64;      // per lane, K or V
    // Row strides in LDS, padded so that the operand reads (16 rows at a time)
    // spread over the banks.
    static constexpr int kStrideK = kRowBytes + 16;
    static constexpr int kStrideV = kRowBytes + (kCache ? 16 : 32);
    static constexpr int kTileBytes = kFewKeys * (kStrideK + kStrideV);
    // the same space holds the wave's output at the end, [16][D + 4] floats
    static constexpr int kMeetBytes = kFewRows * (D + 4) * 4;
    static constexpr int kWaveBytes = kTileBytes > kMeetBytes ? kTileBytes : kMeetBytes;
    static_assert(kFewKeys * kPieces % 64 == 0, "");
};

// Eight codes times `power`, a power of two.
template <int kIn>
__device__ __forceinline__ h8 codes_to(u2 c, float power = 1.f)
{
    h8 out;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if constexpr (kIn == kInBF16) {
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[k], power, false);
            const b2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[k], power, true);
            const h2 x = __builtin_bit_cast(h2, a), y = __builtin_bit_cast(h2, b);
            out[4 * k] = x[0], out[4 * k + 1] = x[1], out[4 * k + 2] = y[0], out[4 * k + 3] = y[1];
        } else {
            const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[k], power, false);
            const h2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[k], power, true);
            out[4 * k] = a[0], out[4 * k + 1] = a[1], out[4 * k + 2] = b[0], out[4 * k + 3] = b[1];
        }
    }
    return out;
}

template <int kIn>
__device__ __forceinline__ f4 mfma16(h8 a, h8 b, f4 c)
{
    if constexpr (kIn == kInBF16)
        return mfma16x16x32_bf16(a, b, c);
    else
        return mfma16x16x32(a, b, c);
}

// Ends a loop body whose last instructions are matrix products: 19 wait states,
// after which their results may be read.  The compiler keeps that distance
// itself, but was seen to miss it where two paths of different length lead from
// the last product to the first read behind the loop (the last register of an
// accumulator was read too early).
__device__ __forceinline__ void products_done()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

// x rounded to the 16-bit type, as raw bits in an f16 register.
template <int kIn>
__device__ __forceinline__ _Float16 to16(float x)
{
    if constexpr (kIn == kInBF16)
        return __builtin_bit_cast(_Float16, (__bf16)x);
    else
        return (_Float16)x;
}

// Its value.
template <int kIn>
__device__ __forceinline__ float from16(_Float16 x)
{
    if constexpr (kIn == kInBF16)
        return (float)__builtin_bit_cast(__bf16, x);
    else
        return (float)x;
}

// Probabilities enter an f16 product times 2^kRaise.  Relative to the row's largest,
// one below 2^-14 would be no normal number of f16 and lose bits, and where many
// keys are alike all of them are off the same way (by 2.4% at 2^-19.6).  With 2^9,
// and the 2^6 by which a maximum may lag behind (many_rows.h), all of f16 is used:
// 11 bits down to 2^-23.  The running maximum is kept that much lower, which costs
// next to nothing.  bf16 has fp32's exponents.
template <int kPV>
constexpr int kRaise = kPV == kInF16 ? 9 : 0;
// A maximum so lowered.  From kLargeScore on fp32's steps no longer hold the 9 (in
// steps of 16 it would be 16, and the largest probability f16's infinity).
constexpr float kLargeScore = 0x1p20f;
template <int kPV>
__device__ __forceinline__ float lowered(float m)
{
    return kRaise<kPV> ? m - (fabsf(m) < kLargeScore ? (float)kRaise<kPV> : 0.f) : m;
}
// a * b, rounded: not to be fused with the subtraction of its own maximum, which
// would leave that rounding (2^7 and more from 2^31 on) in the exponent.
__device__ __forceinline__ float rounded_product(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

__device__ __forceinline__ float sum_xor16_32(float v)
{
    int b = __builtin_bit_cast(int, v);
    auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    v = __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
    b = __builtin_bit_cast(int, v);
    r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}

// Transposed LDS read of bytes (ds_read_b64_tr_b8): within each group of 16
// lanes, lane j returns for k = 0..7 byte j % 8 of the 8 bytes that group lane
// 2k + j / 8 addresses (checked on the GPU).  With group lane s at row s / 2,
// columns 8 (s % 2) .. + 7, lane j receives column j of 8 rows.
__device__ __forceinline__ u2 lds_read_tr8(const uint8_t *p)
{
    return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)p));
}

// The four outputs of an O^T accumulator, as they are stored.
template <int kIn>
__device__ __forceinline__ void store4(void *O, int64_t at, f4 v)
{
    const h4 x = {to16<kIn>(v[0]), to16<kIn>(v[1]), to16<kIn>(v[2]), to16<kIn>(v[3])};
    *reinterpret_cast<h4 *>(reinterpret_cast<_Float16 *>(O) + at) = x;
}

// Natural log-sum-exp of a row with sum l relative to 2^m.
__device__ __forceinline__ float natural_lse(float m, float l)
{
    return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// The partial results of a row: n of them at rows first, first + stride, ...  Each
// is an output and a sum l relative to 2^(m + kRaise), m its (lowered) maximum.
struct PartRows {
    int64_t first, stride;
    int n;
};

// Joins a row's partial results (those of x, then those of y) and stores it at
// row `out` of O and lse.  kSplit: the whole workgroup of 256 threads does it,
// each group of D / 4 threads (four columns each) every G-th piece, the groups'
// states meeting in LDS; else one group of D / 4 threads does it alone, `c` its
// thread's first column.  Four pieces' loads are in flight together. With few
// rows the pieces' loads one behind the other are what a join waits for, with
// many the workgroups and what they read: of 128 values, 1,024 rows of 17 pieces
// took 8.8 us split and 14.6 by one group, 2,048 rows 8.4 and 9.2, 4,096 rows 9.2
// and 8.4, 8,192 rows of 9 pieces 14.5 and 10.1.
template <int D, int kIn, int kPV, bool kSplit>
__device__ __forceinline__ void join_row(const float *part_o, const float *part_ml,
                                         const PartRows &x, const PartRows &y, int64_t out,
                                         void *O, float *lse)
{
    constexpr int kGroup = D / 4, kAhead = 4;
    constexpr int kGroups = kSplit ? 256 / kGroup : 1;
    __shared__ float s_ml[kGroups][2];
    __shared__ __attribute__((aligned(16))) float s_o[kSplit ? kGroups : 1][kSplit ? D : 4];
    const int group = kSplit ? (int)threadIdx.x / kGroup : 0;
    const int c = (int)threadIdx.x % kGroup * 4;
    const int n = x.n + y.n;
    float m = -INFINITY, l = 0.f;
    f4 o = f4{0.f, 0.f, 0.f, 0.f};
    for (int p = group; p < n && group < kGroups; p += kGroups * kAhead) {
        f4 po[kAhead];
        float pm[kAhead], pl[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = min(p + k * kGroups, n - 1);
            const int64_t row =
                at < x.n ? x.first + x.stride * at : y.first + y.stride * (at - x.n);
            pm[k] = part_ml[2 * row];
            pl[k] = part_ml[2 * row + 1];
            po[k] = *reinterpret_cast<const f4 *>(part_o + row * D + c);
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (p + k * kGroups >= n) pm[k] = -INFINITY;
            top = fmaxf(top, pm[k]);
        }
        const float ref = top == -INFINITY ? 0.f : top;
        const float f = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= f;
        o *= f;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float w = __builtin_amdgcn_exp2f(pm[k] - ref);
            l += w * pl[k];
            o += w * po[k];
        }
    }
    if constexpr (kSplit) {
        if (group < kGroups) {
            if (c == 0) {
                s_ml[group][0] = m;
                s_ml[group][1] = l;
            }
            *reinterpret_cast<f4 *>(&s_o[group][c]) = o;
        }
        __syncthreads();
        if (threadIdx.x >= kGroup) return;
        float top = s_ml[0][0];
#pragma unroll
        for (int k = 1; k < kGroups; ++k) top = fmaxf(top, s_ml[k][0]);
        const float ref = top == -INFINITY ? 0.f : top;
        m = top;
        l = 0.f;
        o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const float w = __builtin_amdgcn_exp2f(s_ml[k][0] - ref);
            l += w * s_ml[k][1];
            o += w * *reinterpret_cast<const f4 *>(&s_o[k][c]);
        }
    }
    store4<kIn>(O, out * D + c, o * (l == 0.f ? 0.f : 1.f / l));
    if (c == 0) lse[out] = natural_lse(m + kRaise<kPV>, l);
}

// Rows up to which a workgroup joins one.
constexpr int64_t kSplitJoins = 2048;

template <int D, int kIn, bool kCache>
__device__ __forceinline__ void few_rows(const FewArgs &a, const FewItem &it)
{
    using T = FewTile<D, kCache>;
    constexpr int kPV = kCache ? kInF16 : kIn;  // type of the value product
    __shared__ __attribute__((aligned(16))) uint8_t s_tile[kFewWaves][T::kWaveBytes];
    __shared__ float s_ml[kFewWaves][2][kFewRows];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    uint8_t *const tile_k = s_tile[wave];
    uint8_t *const tile_v = s_tile[wave] + kFewKeys * T::kStrideK;

    // Q as the second operand: row i, elements 32 c + 8 g .. + 7
    h8 q[D / 32];
    {
        const int64_t at = query_row(a.q, it.head, it.row + (i < it.rows ? i : 0)) * D + 8 * g;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            u4 x = *reinterpret_cast<const u4 *>(reinterpret_cast<const _Float16 *>(a.Q) + at +
                                                 32 * c);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = i < it.rows ? x[k] ^ a.flip : 0u;
            q[c] = __builtin_bit_cast(h8, x);
        }
    }
    // keys that this lane's row sees
    const int limit =
        it.causal ? max(it.begin, min(it.end, it.limit + (it.first + i) / a.q.g)) : it.end;
    const int least = it.causal ? max(it.begin, min(it.end, it.limit + it.first / a.q.g)) : it.end;

    f4 o[D / 16];
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[t] = f4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;  // maximum, lowered by kRaise
    int ref = 0;  // cache: this row's o holds multiples of 2^(ref - 127)

    u4 kr[T::kLoads], vr[T::kLoads];
    uint32_t ke[2] = {0, 0}, ve[2] = {0, 0};
    int pages[2] = {0, 0};  // of the tile in kr, vr; -1: none

    auto load = [&](int t) {
        if constexpr (kCache) {
            int64_t base[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int pos = t + 16 * h;
                const int n = pos >> a.page_shift;
                int page = pos < it.end && n < it.table_len ? it.table[n] : -1;
                page = __builtin_amdgcn_readfirstlane(page);
                pages[h] = page >= 0 && page < a.n_pages ? page : -1;
                // (a page that is none reads page 0, whose keys are left out)
                base[h] = ((((int64_t)max(pages[h], 0) * a.n_kv + it.head) << a.page_shift) +
                           (pos & ((1 << a.page_shift) - 1)));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ke[h] = *reinterpret_cast<const uint32_t *>(a.k_exp + base[h] + 4 * g);
                ve[h] = *reinterpret_cast<const uint32_t *>(a.v_exp + base[h] + 4 * g);
            }
#pragma unroll
            for (int j = 0; j < T::kLoads; ++j) {
                const int f = lane + 64 * j, row = f / T::kPieces;
                const int64_t at = (row < 16 ? base[0] : base[1] - 16) * D + f * 16;
                kr[j] = *reinterpret_cast<const u4 *>(a.k + at);
                vr[j] = *reinterpret_cast<const u4 *>(a.v + at);
            }
        } else {
#pragma unroll
            for (int j = 0; j < T::kLoads; ++j) {
                const int f = lane + 64 * j, row = f / T::kPieces;
                // (rows behind the range read its last one, which is left out)
                const int64_t r = it.key + min(t + row, it.end - 1);
                const int64_t at = (r * a.n_kv + it.head) * (2 * D) + (f - row * T::kPieces) * 16;
                kr[j] = *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(a.K) + at);
                vr[j] = *reinterpret_cast<const u4 *>(reinterpret_cast<const uint8_t *>(a.V) + at);
            }
        }
    };

    int t = it.begin + kFewKeys * wave;
    constexpr int kStep = kFewKeys * kFewWaves;
    if (t < it.end) load(t);
    for (; t < it.end; t += kStep) {
        const bool ok0 = !kCache || pages[0] >= 0, ok1 = !kCache || pages[1] >= 0;
        const bool whole = t + kFewKeys <= least && ok0 && ok1;
        const int keys0 = ok0 ? min(it.end - t, 16) : 0, keys1 = ok1 ? min(it.end - t, 32) : 0;
        const uint32_t kx[2] = {ke[0], ke[1]};
        uint32_t vx[2] = {ve[0], ve[1]};
        tile_fence<kFewWaves>();
#pragma unroll
        for (int j = 0; j < T::kLoads; ++j) {
            const int f = lane + 64 * j, row = f / T::kPieces, c = f - row * T::kPieces;
            // values that are left out have to be finite: 0 times them is added
            if (!whole && row >= (row < 16 ? keys0 : keys1)) vr[j] = u4{0, 0, 0, 0};
            *reinterpret_cast<u4 *>(tile_k + row * T::kStrideK + c * 16) = kr[j];
            *reinterpret_cast<u4 *>(tile_v + row * T::kStrideV + c * 16) = vr[j];
        }
        tile_fence<kFewWaves>();
        if (t + kStep < it.end) load(t + kStep);

        f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t *row = tile_k + (16 * h + i) * T::kStrideK;
                h8 k;
                if constexpr (kCache)
                    k = codes_to<kIn>(*reinterpret_cast<const u2 *>(row + 32 * c + 8 * g));
                else
                    k = *reinterpret_cast<const h8 *>(row + 64 * c + 16 * g);
                s[h] = mfma16<kIn>(k, q[c], s[h]);
            }
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = rounded_product(s[e >> 2][e & 3], a.sl2);
            if constexpr (kCache)
                x[e] = __builtin_ldexpf(x[e], (int)((kx[e >> 2] >> (8 * (e & 3))) & 255) - 127);
        }
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = 16 * (e >> 2) + 4 * g + (e & 3);
                if (t + key >= limit || key >= (e < 4 ? keys0 : keys1)) {
                    x[e] = -INFINITY;
                    // (no power of its own: a row's sums are relative to what it sees)
                    if (kCache) vx[e >> 2] &= ~(255u << (8 * (e & 3)));
                }
            }
        }
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
        mx = max_xor32(max_xor16(mx));
        const float m_new = fmaxf(m_run, lowered<kPV>(mx));
        const float m_ref = m_new == -INFINITY ? 0.f : m_new;  // (no key yet)
        float alpha = __builtin_amdgcn_exp2f(m_run - m_ref);
        bool rescale = m_new > m_run;
        m_run = m_new;
        float p[8], sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(x[e] - m_ref);
            sum += p[e];
        }
        l_run = l_run * alpha + sum;
        if constexpr (kCache) {
            int top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                top = max(top, (int)((vx[e >> 2] >> (8 * (e & 3))) & 255));
            auto r = __builtin_amdgcn_permlane16_swap(top, top, false, false);
            top = max((int)r[0], (int)r[1]);
            r = __builtin_amdgcn_permlane32_swap(top, top, false, false);
            top = max((int)r[0], (int)r[1]);
            if (top > ref) {
                alpha = __builtin_ldexpf(alpha, ref - top);
                ref = top;
                rescale = true;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                p[e] = __builtin_ldexpf(p[e], (int)((vx[e >> 2] >> (8 * (e & 3))) & 255) - ref);
        }
        if (__ballot(rescale)) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= alpha;
        }
        h8 pf;
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[e] = to16<kPV>(p[e]);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            h8 vt;
            if constexpr (kCache) {
                // rows 4 g .. + 3 of both halves, columns 16 d ..
                const int row = (i >> 1 & 3) + 4 * g + (i >> 3) * 16;
                vt = codes_to<kInF16>(
                    lds_read_tr8(tile_v + row * T::kStrideV + 16 * d + 8 * (i & 1)));
            } else {
                const _Float16 *v = reinterpret_cast<const _Float16 *>(
                    tile_v + (4 * g + (i >> 2)) * T::kStrideV + 32 * d + 8 * (i & 3));
                vt = cat44(lds_read_tr(v), lds_read_tr(v + 16 * T::kStrideV / 2));
            }
            o[d] = mfma16<kPV>(vt, pf, o[d]);
        }
        products_done();
    }

    // the four waves' states meet: scaled to the common maximum and summed
    constexpr float kLower = 1.f / (1 << kRaise<kPV>);
    const float l_all = sum_xor16_32(l_run) * kLower;
    float *const mine = reinterpret_cast<float *>(s_tile[wave]);
    tile_fence<kFewWaves>();
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
        if (kCache) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[d][k] = __builtin_ldexpf(o[d][k], ref - 127 - kRaise<kPV>);
        } else {
            o[d] *= kLower;
        }
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
        *reinterpret_cast<f4 *>(mine + i * (D + 4) + 16 * d + 4 * g) = o[d];
    if (g == 0) {
        s_ml[wave][0][i] = m_run;
        s_ml[wave][1][i] = l_all;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kFewRows * D / 4; e += 64 * kFewWaves) {
        const int r = e / (D / 4), c = (e - r * (D / 4)) * 4;
        if (r >= it.rows) continue;
        float m = s_ml[0][0][r];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) m = fmaxf(m, s_ml[w][0][r]);
        const float m_ref = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f4 sum = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_ml[w][0][r] - m_ref);
            l += f * s_ml[w][1][r];
            sum += f * *reinterpret_cast<const f4 *>(
                           reinterpret_cast<const float *>(s_tile[w]) + r * (D + 4) + c);
        }
        if (it.part >= 0) {
            *reinterpret_cast<f4 *>(a.part_o + (it.part + r) * D + c) = sum;
            if (c == 0) {
                a.part_ml[2 * (it.part + r)] = m;
                a.part_ml[2 * (it.part + r) + 1] = l;
            }
        } else {
            const int64_t at = query_row(a.q, it.head, it.row + r);
            store4<kIn>(a.O, at * D + c, sum * (l == 0.f ? 0.f : 1.f / l));
            if (c == 0) a.lse[at] = natural_lse(m + kRaise<kPV>, l);
        }
    }
}

}  // namespace f3s
