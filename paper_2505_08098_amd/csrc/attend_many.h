// Attention of many query rows to the shared prefix of the 8-bit cache (the
// first of f3s_cache_attend's passes where the batch has more than a few rows).
//
// The kernel of many_rows.h with another way into LDS: a tile's codes wait in
// registers and are widened as they are stored, once for the 128 rows of the
// workgroup, K to the queries' type and V to f16.  The vector unit is what bounds
// it (each exponential, maximum and sum costs the cycles that 1/2 product does),
// so the powers of two ride on that conversion: a key's relative to the tile's
// largest, which multiplies the scores within the exponential's own fused
// operation, a value's relative to the largest that the workgroup has met, which
// the sums are multiples of.  A code has four bits, so the widened value is exact
// unless its row is 2^15 times smaller than that largest one (f16; 2^117 in
// bf16); then it is off by at most 2^-25 of the largest power, which is no more
// than the probabilities' own rounding leaves.
//
// 512 rows of a key head, 16,384 keys, 8 key heads of 128: 54 us, 635 TFLOP/s; a
// tile of 64 keys takes 2.7 us, the beginning and the partial results 14.
#pragma once

#include "attend.h"
#include "many_rows.h"

namespace f3s {

// Keys that one workgroup walks at most: its pages' numbers wait in LDS.
constexpr int kMostChunk = 4096;

// Keys of a tile (the codes on their way leave no room for 64 of 128 values).
constexpr int code_keys(int d) { return d <= 128 ? 64 : 32; }
constexpr int code_sets(int d) { return code_keys(d) == 64 ? 1 : 2; }
constexpr int prefix_waves(int d) { return d <= 64 ? 3 : d <= 128 ? 2 : 1; }

// One of the two buffers of a tile of cached keys.
template <int D>
struct CodeTile {
    using T = ManyTile<D, code_keys(D)>;
    __attribute__((aligned(16))) uint8_t k[T::kBytes], v[T::kBytes];
};

// Largest of the lower and of the upper halves of a wave's numbers, by lane moves
// of the vector unit (through LDS they would hold up the wave that every other
// one waits for).
__device__ __forceinline__ uint32_t wave_max2(uint32_t v)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    auto larger = [](uint32_t x, uint32_t y) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
            __builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
    };
    v = larger(v, __builtin_amdgcn_mov_dpp(v, 0x121, 0xF, 0xF, true));  // row_ror:1
    v = larger(v, __builtin_amdgcn_mov_dpp(v, 0x122, 0xF, 0xF, true));
    v = larger(v, __builtin_amdgcn_mov_dpp(v, 0x124, 0xF, 0xF, true));
    v = larger(v, __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true));
    auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = larger(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return __builtin_amdgcn_readfirstlane(larger(r[0], r[1]));
}

// 2^e for e <= 0, at least 2^-126.
__device__ __forceinline__ float power_of(int e)
{
    return __builtin_bit_cast(float, (max(e, -126) + 127) << 23);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, prefix_waves(D)) void k_attend_prefix(AttendArgs a)
{
    using T = ManyTile<D, code_keys(D)>;
    constexpr int kKeys = T::kRows, kBlocks = kKeys / 32;
    constexpr int kCodes = D / 16;  // 16-byte pieces of a row of codes
    constexpr int kLoads = (kKeys * kCodes + kManyThreads - 1) / kManyThreads;
    constexpr bool kEven = kKeys * kCodes % kManyThreads == 0;
    __shared__ CodeTile<D> s0, s1;
    __shared__ int32_t s_pages[kMostChunk / 16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int tile = (int)blockIdx.x % a.prefix_blocks, sh = (int)blockIdx.x / a.prefix_blocks;
    const int head = sh % a.few.n_kv, split = sh / a.few.n_kv;
    const int64_t all = (int64_t)a.rows * a.n_seqs;  // rows of the key head
    const int rows = (int)(all - (int64_t)tile * kManyRows < kManyRows
                               ? all - (int64_t)tile * kManyRows : kManyRows);
    const int begin = split * a.prefix_chunk, end = min(a.prefix_len, begin + a.prefix_chunk);
    const int shift = a.few.page_shift;
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < rows;
    const bool busy = 32 * wave < rows;

    h8 q[D / 16];
    load_rows32<D>(q, a.few.Q,
                   query_row(a.few.q, head, (int64_t)tile * kManyRows + (there ? mine : 0)),
                   there, a.few.flip, lane);
    const int page0 = begin >> shift;
    for (int i = threadIdx.x; i < ((end - 1) >> shift) - page0 + 1; i += kManyThreads)
        s_pages[i] = a.prefix[page0 + i];
    __syncthreads();

    f16v o[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = zero16();
    float m_run = -INFINITY, l_run = 0.f;  // maximum, lowered by kRaise
    uint64_t large = 0;  // lanes where it is from kLargeScore on
    int ref = 0;  // o holds multiples of 2^(ref - 127)

    constexpr int kSets = code_sets(D);
    u4 kr[kSets][kLoads], vr[kSets][kLoads];
    bool ok[kSets];  // whether the key that this lane looks after is there
    uint32_t ke[kSets], ve[kSets];
    // Of the tiles in LDS: the keys that are there, a bit each, what their scores
    // are multiplied by, and the power that their values are relative to.
    uint64_t keys[2];
    float times[2];
    int top[2], most = 0;
    // Row of the cache of a key of the range; of one that is not there any row.
    auto place = [&](int key, bool *there) -> int64_t {
        const int page = s_pages[(min(key, end - 1) >> shift) - page0];
        *there = key < end && (unsigned)page < (unsigned)a.few.n_pages;
        return (((int64_t)(*there ? page : 0) * a.few.n_kv + head) << shift) +
               (key & ((1 << shift) - 1));
    };
    auto fetch = [&](int t, auto b) {
        constexpr int w = kSets > 1 ? decltype(b)::kIndex : 0;
        const int first = begin + kKeys * t;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int f = (int)threadIdx.x + kManyThreads * j;
            const int row = kEven ? f / kCodes : min(f / kCodes, kKeys - 1);
            bool there;
            const int64_t at = place(first + row, &there) * D + f % kCodes * 16;
            kr[w][j] = *reinterpret_cast<const u4 *>(a.few.k + at);
            vr[w][j] = *reinterpret_cast<const u4 *>(a.few.v + at);
        }
        const int64_t r = place(first + (int)threadIdx.x % kKeys, &ok[w]);
        ke[w] = a.few.k_exp[r];
        ve[w] = a.few.v_exp[r];
    };
    auto put = [&](auto b) {
        constexpr int w = kSets > 1 ? decltype(b)::kIndex : 0;
        constexpr int at = b.kIndex;
        CodeTile<D> &to = at ? s1 : s0;
        const int mine = ok[w] ? (int)(ke[w] | ve[w] << 16) : -1;  // its powers, or -1
        keys[at] = __ballot(mine >= 0);  // (of 32 keys: each twice)
        const uint32_t tops = wave_max2(mine < 0 ? 0 : mine);
        const int key_top = tops & 255;
        most = max(most, (int)(tops >> 16));
        top[at] = most;
        times[at] = fminf(__builtin_ldexpf(a.few.sl2, key_top - 127), 0x1.fffffep127f);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int f = (int)threadIdx.x + kManyThreads * j, row = f / kCodes;
            const int its = __builtin_amdgcn_ds_bpermute(4 * row, mine);
            if (!kEven && row >= kKeys) continue;
            const int c = f % kCodes, sw = T::swizzle(row & 31);
            // (a value that is left out has to be finite: 0 times it is added)
            if (its < 0) vr[w][j] = u4{0, 0, 0, 0};
            const float kp = power_of(its < 0 ? 0 : (its & 255) - key_top);
            const float vp = power_of(its < 0 ? 0 : (its >> 16) - most);
            const u2 klo = {kr[w][j][0], kr[w][j][1]}, khi = {kr[w][j][2], kr[w][j][3]};
            const u2 vlo = {vr[w][j][0], vr[w][j][1]}, vhi = {vr[w][j][2], vr[w][j][3]};
            uint8_t *pk = to.k + row * T::kStride, *pv = to.v + row * T::kStride;
            *reinterpret_cast<h8 *>(pk + ((2 * c) ^ sw) * 16) = codes_to<kIn>(klo, kp);
            *reinterpret_cast<h8 *>(pk + ((2 * c + 1) ^ sw) * 16) = codes_to<kIn>(khi, kp);
            *reinterpret_cast<h8 *>(pv + ((2 * c) ^ sw) * 16) = codes_to<kInF16>(vlo, vp);
            *reinterpret_cast<h8 *>(pv + ((2 * c + 1) ^ sw) * 16) = codes_to<kInF16>(vhi, vp);
        }
    };
    auto work = [&](auto b) {
        if (!busy) return;
        const CodeTile<D> &from = b.kIndex ? s1 : s0;
        f16v s[kBlocks];
#pragma unroll
        for (int h = 0; h < kBlocks; ++h) s[h] = zero16();
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
#pragma unroll
            for (int h = 0; h < kBlocks; ++h)
                s[h] = mfma32<kIn>(T::rows32(from.k, 32 * h, c, lane), q[c], s[h]);
        }
        float by = times[b.kIndex];
        const uint64_t all = keys[b.kIndex];
        if (kBlocks > 1 ? ~all : ~(uint32_t)all) {
#pragma unroll
            for (int h = 0; h < kBlocks; ++h) {
                const uint32_t mask = (uint32_t)(all >> 32 * h) >> (4 * (lane >> 5));
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[h][e] = mask >> (8 * (e >> 2) + (e & 3)) & 1 ? s[h][e] * by : -INFINITY;
            }
            by = 1.f;  // (0 times infinity would be NaN)
        }
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < 16 * kBlocks; ++e) mx = fmaxf(mx, s[e >> 4][e & 15]);
        mx = rounded_product(max_xor32(mx), by);
        // (a maximum that has grown by less than 2^6 is not worth the products: the
        // probabilities may as well be 64 times larger, with the same 11 bits)
        if (__ballot(mx - m_run > kRaise<kInF16> + 6.f) || top[b.kIndex] > ref) {
            const float m_new = fmaxf(m_run, lowered<kInF16>(mx));
            float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            l_run *= alpha;
            alpha = __builtin_ldexpf(alpha, ref - top[b.kIndex]);
            ref = top[b.kIndex];
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= alpha;
            m_run = m_new;
            large = __ballot(fabsf(m_run) >= kLargeScore && m_run > -INFINITY);
        }
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;
        if (large) {  // (see rounded_product)
#pragma unroll
            for (int e = 0; e < 16 * kBlocks; ++e)
                s[e >> 4][e & 15] = rounded_product(s[e >> 4][e & 15], by);
            by = 1.f;
        }
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < kBlocks; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[h][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][e], by, -m_ref));
                sum += s[h][e];
            }
        l_run += sum;
#pragma unroll
        for (int c = 0; c < 2 * kBlocks; ++c) {
            const h8 p = pack8<kInF16>(s[c >> 1], c & 1);
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                o[d] = mfma32<kInF16>(T::cols32(from.v, 16 * c, 32 * d, lane), p, o[d]);
        }
        products_done();
    };
    const int n = (end - begin + kKeys - 1) / kKeys;
    auto step = [&](int t, auto here, auto next) {
        __syncthreads();  // tile t is there, and nobody reads the other buffer
        if (t + 1 < n) {
            put(next);
            fetch(min(t + 1 + kSets, n - 1), next);
        }
        work(here);
    };
    fetch(0, Buffer<0>());
    if (kSets > 1) fetch(min(1, n - 1), Buffer<1>());
    put(Buffer<0>());
    fetch(min(kSets, n - 1), Buffer<0>());
    for (int t = 0; t < n; t += 2) {
        step(t, Buffer<0>(), Buffer<1>());
        if (t + 1 < n) step(t + 1, Buffer<1>(), Buffer<0>());
    }

    const float l = __builtin_ldexpf(sum_xor32(l_run), -kRaise<kInF16>);
    const int64_t part = a.prefix_part + ((int64_t)split * a.few.n_kv + head) * all +
                         (int64_t)tile * kManyRows + 32 * wave;
    uint8_t *const lds = wave == 0 ? s0.k : wave == 1 ? s0.v : wave == 2 ? s1.k : s1.v;
    __syncthreads();  // nobody reads the tiles
    store_part32<D, T::kBytes / 128 / 32 * 32>(
        lds, o, __builtin_ldexpf(1.f, ref - 127 - kRaise<kInF16>), a.few.part_o + part * D, D,
        rows - 32 * wave, lane);
    if (there && lane < 32) {
        a.few.part_ml[2 * (part + lane)] = m_run;
        a.few.part_ml[2 * (part + lane) + 1] = l;
    }
}

template <int D, int kIn>
hipError_t launch_attend_prefix_d(const AttendArgs &a, hipStream_t s)
{
    const int64_t grid = (int64_t)a.prefix_splits * a.few.n_kv * a.prefix_blocks;
    k_attend_prefix<D, kIn><<<(unsigned)grid, kManyThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace f3s
