// Attention over the 8-bit cache with a mask: a sliding window with sinks
// (f3s_cache_attend_window) or the ancestors in a tree of drafted tokens
// (f3s_cache_attend_tree).  Few query rows of a key head go through few_rows.h, 16 at a
// time; many through the kernel here, 128 or 256 at a time.
//
// The kernel of many rows is that of attend_many.h for tiles of keys that every row of the
// workgroup sees: their codes are widened once for all rows, times powers of two relative
// to the tile's largest (K) and to the largest so far (V).  In tiles that some rows do not
// see all of (the window's edge, the diagonal, the tree) such a common power would let a
// key that a row does not see take bits from those it sees.  There codes are widened as
// they are, and the powers multiply each score and each probability, relative to the
// largest that the row itself has seen.  They have a walk of their own, behind that of the
// others, so that the sums' power is the workgroup's until then and the row's from there
// on (and since both kinds in one loop would spill).  A row's result is its own, bit by
// bit, whatever the others see.
//
// 2 x 2,000 tokens over a window of 4,000, 16 heads of 128 over 4: 159 to 166 us by card (770
// to 800 TFLOP/s); the matrix units are busy 31% of the cycles and the vector unit issues in
// 42%, by turns, since the eight waves of a compute unit meet at a barrier every tile.  16
// trees of 63 tokens over 500 to 8,192 own keys and 2,001 shared ones, 32 heads over 8: 160 to
// 166 us, of which the join takes 14 (30% and 47%; the longest pieces have 44 units where 34
// would be even).  By 16 rows bytes bound it: one token of 64 sequences over a window of
// 4,096, 8 key heads of 128, 90 us, 5.5 TB/s.
#pragma once

#include "attend_many.h"

namespace f3s {

// Workgroups of w waves that a compute unit holds: what the registers leave room for.
constexpr int own_groups(int d, int w) { return w == 8 ? 1 : d <= 64 ? 3 : d <= 128 ? 2 : 1; }
// Whether there is a kernel of 256 rows (two waves per SIMD as one workgroup).
constexpr bool own_wide(int d) { return d > 64 && d <= 128; }

// A number that is the same for all lanes, where the compiler might not see it.
__device__ __forceinline__ int32_t uniform(int32_t x)
{
    return __builtin_amdgcn_readfirstlane(x);
}

// Keys that some row of a block sees, in a window: tokens first .. last of a sequence of
// `keys` cached ones whose first new token stands at `base`.
__device__ __forceinline__ WindowKeys own_window(const WindowRule &rule, int32_t base, int first,
                                                 int last, int32_t keys)
{
    WindowKeys k = window_keys(rule, base + first, base + last, 16);
    k.end = min(k.end, keys);
    k.near = min(k.near, k.end);
    k.far = min(k.far, keys);
    return k;
}

// Piece `split` of a list of n places, in places.
struct Places {
    int32_t begin, end;
};
__device__ __forceinline__ Places places_of(int32_t n, int32_t split, int32_t splits)
{
    const int32_t units = units_of(n);
    return {item_unit(units, split, splits) * kUnit,
            min(n, item_unit(units, split + 1, splits) * kUnit)};
}

template <int D, int kIn>
__global__ __launch_bounds__(64 * kFewWaves, few_waves(D, true)) void k_attend_window(
    AttendArgs a)
{
    FewItem it = {};
    const int rb = (int)blockIdx.x % a.row_blocks, ih = (int)blockIdx.x / a.row_blocks;
    it.head = ih % a.few.n_kv;
    const int i = ih / a.few.n_kv, seq = i / a.splits, split = i - seq * a.splits;
    if (split == 0 && it.head == 0 && rb == 0 && threadIdx.x == 0 && !a.direct)
        a.desc[seq] = int2{i, a.splits};
    it.row = (int64_t)seq * a.rows + rb * kFewRows;
    it.rows = min(kFewRows, a.rows - rb * kFewRows);
    it.first = rb * kFewRows;
    it.table = a.table + (int64_t)seq * a.max_pages;
    it.table_len = a.max_pages;
    const int32_t keys = cache_keys(a.lens[seq], (int64_t)a.max_pages << a.few.page_shift);
    const int32_t base = (int32_t)cache_position(a.lens[seq], a.n_new, 0);
    it.limit = base + 1;
    it.keys = own_window(a.rule, base, it.first / a.few.q.g,
                         (it.first + it.rows - 1) / a.few.q.g, keys);
    const Places p = places_of(window_length(it.keys), split, a.splits);
    it.begin = p.begin;
    it.end = p.end;
    it.part = a.direct ? -1 : ((int64_t)i * a.few.n_kv + it.head) * a.rows + rb * kFewRows;
    few_rows<D, kIn, true, kWindowMask>(a.few, it, a.rule);
}

template <int D, int kIn>
__global__ __launch_bounds__(64 * kFewWaves, few_waves(D, true)) void k_attend_tree(AttendArgs a)
{
    __shared__ uint32_t s_bits[kFewRows][kTreeWords];
    __shared__ int32_t s_parents[kTreeTokens];
    const int wg = (int)blockIdx.x, n_prefix = few_prefix(a);
    FewItem it;
    if (wg < n_prefix) {
        it = prefix_item(a, wg);
        it.base = kMostTokens;  // (all of it lies before the tree)
    } else {
        it = own_keys_item(a, wg - n_prefix);
    }
    if (it.rows == 0) return;
    if (it.end > it.base || it.base < 0) {
        const int64_t seq = it.row / a.rows;
        tree_bits<kFewRows>(s_bits, s_parents, a.parents + seq * a.n_new, a.n_new, it.first,
                            a.few.q.g, it.base);
    } else if (threadIdx.x < kFewRows) {
        s_bits[threadIdx.x][0] = ~0u;  // (all that is read where the keys end before the tree)
    }
    __syncthreads();
    few_rows<D, kIn, true, kTreeMask>(a.few, it, {}, s_bits);
}

// Item i where the own keys are divided into at most a.own_items items (at least as many
// as sequences) of as few units as that allows: a round of the compute units ends when
// its longest item does.  16 trees of 63 tokens behind 8 to 128 units, 32 heads of 128
// over 8: 178 us a call where shares happen to fill a round, 190 to 219 where not.
__device__ __forceinline__ OwnItem fitted_item(const AttendArgs &a, int i)
{
    const int lane = threadIdx.x & 63;
    const int64_t cap = (int64_t)a.max_pages << a.few.page_shift;
    if (a.whole) return own_item(a, i);
    // units of this lane's sequence of the first 64, and of any
    const int mine =
        lane < a.n_seqs ? units_of(cache_keys(a.lens[lane], cap)) : 0;
    auto units = [&](int b) {
        return b < 64 ? mine : units_of(cache_keys(a.lens[b], cap));
    };
    int total = 0, longest = 0;
    for (int b = lane; b < a.n_seqs; b += 64) {
        total += units(b);
        longest = max(longest, units(b));
    }
    total = uniform(wave_sum(total));
#pragma unroll
    for (int s = 1; s < 64; s *= 2) longest = max(longest, __shfl_xor(longest, s));
    int low = units_per_item(total, a.own_items), high = max(uniform(longest), low);
    while (low < high) {
        const int per = low + (high - low) / 2;
        int items = 0;
        for (int b = lane; b < a.n_seqs; b += 64) items += items_of(units(b), per);
        if (uniform(wave_sum(items)) <= a.own_items)
            high = per;
        else
            low = per + 1;
    }
    return own_item_at(a, i, low);
}

// W waves, 32 rows each.
template <int D, int kIn, int kMask, int W>
__global__ __launch_bounds__(64 * W, W / 4 * own_groups(D, W)) void k_attend_own(AttendArgs a)
{
    using T = ManyTile<D, code_keys(D)>;
    constexpr int kThreads = 64 * W, kRows = 32 * W;
    constexpr int kKeys = T::kRows, kBlocks = kKeys / 32;
    constexpr int kCodes = D / 16;  // 16-byte pieces of a row of codes
    constexpr int kLoads = (kKeys * kCodes + kThreads - 1) / kThreads;
    constexpr bool kEven = kKeys * kCodes % kThreads == 0;
    constexpr bool kTree = kMask == kTreeMask;
    __shared__ CodeTile<D> s0, s1;
    // the powers of a tile's keys (K | V << 8)
    __shared__ __attribute__((aligned(16))) uint32_t s_powers[2][kKeys];
    __shared__ uint32_t s_bits[kTree ? kRows : 1][kTreeWords];
    __shared__ int32_t s_parents[kTree ? kTreeTokens : 1];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // a tree's prefix: workgroups behind those of the own keys
    const int n_own = a.own_items * a.few.n_kv * a.row_blocks;
    const bool prefix = kTree && (int)blockIdx.x >= n_own;
    const int wg = (int)blockIdx.x - (prefix ? n_own : 0);
    const int blocks = prefix ? a.prefix_blocks : a.row_blocks;
    const int rb = wg % blocks, ih = wg / blocks;
    const int head = ih % a.few.n_kv, i = ih / a.few.n_kv;
    const int first = rb * kRows, rows = min(kRows, a.rows * (prefix ? a.n_seqs : 1) - first);
    const int shift = a.few.page_shift, g = a.few.q.g;
    int seq, begin, end;
    int32_t base;
    WindowKeys list;
    if (prefix) {
        // all sequences' rows as one's, and all keys ahead of its tree
        seq = 0;
        base = kMostTokens;
        list = {0, 0, a.prefix_len};
        begin = i * a.prefix_chunk;
        end = min(a.prefix_len, begin + a.prefix_chunk);
    } else if constexpr (kTree) {
        const OwnItem o = fitted_item(a, i);
        if (o.seq < 0) return;
        seq = o.seq;
        base = (int32_t)cache_position(uniform(a.lens[seq]), a.n_new, 0);
        if (i == o.first && head == 0 && rb == 0 && threadIdx.x == 0 && !a.direct)
            a.desc[seq] = int2{o.first, o.items};
        list = {0, 0, o.keys};
        begin = item_unit(o.units, i - o.first, o.items) * kUnit;
        end = min(o.keys, item_unit(o.units, i - o.first + 1, o.items) * kUnit);
    } else {
        seq = i / a.splits;
        const int split = i - seq * a.splits;
        const int32_t len = uniform(a.lens[seq]);
        if (split == 0 && head == 0 && rb == 0 && threadIdx.x == 0 && !a.direct)
            a.desc[seq] = int2{i, a.splits};
        base = (int32_t)cache_position(len, a.n_new, 0);
        list = own_window(a.rule, base, first / g, (first + rows - 1) / g,
                          cache_keys(len, (int64_t)a.max_pages << shift));
        const Places p = places_of(window_length(list), split, a.splits);
        begin = p.begin;
        end = p.end;
    }
    const int32_t *const table = prefix ? a.prefix : a.table + (int64_t)seq * a.max_pages;
    const int64_t row0 = (int64_t)seq * a.rows + first;  // of the key head's rows
    // first partial row
    const int64_t part0 =
        prefix ? a.prefix_part + ((int64_t)i * a.few.n_kv + head) * a.rows * a.n_seqs + first
               : ((int64_t)i * a.few.n_kv + head) * a.rows + first;
    const int mine = 32 * wave + (lane & 31);
    const bool there = mine < rows;
    const bool busy = 32 * wave < rows;
    // positions of the block's first and last token, and of this lane's
    const int p_first = base + first / g, p_last = base + (first + rows - 1) / g;
    const int p_mine = base + (first + (there ? mine : 0)) / g;

    h8 q[D / 16];
    load_rows32<D>(q, a.few.Q, query_row(a.few.q, head, row0 + (there ? mine : 0)), there,
                   a.few.flip, lane);
    if (kTree && !prefix)
        tree_bits<kRows>(s_bits, s_parents, a.parents + (int64_t)seq * a.n_new, a.n_new,
                             first, g, base);

    f16v o[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = zero16();
    float m_run = -INFINITY, l_run = 0.f;  // maximum, lowered by kRaise
    uint64_t large = 0;  // lanes where it is from kLargeScore on
    int ref = 0;         // this row's o holds multiples of 2^(ref - 127)

    // The tiles of the walk, and the next one behind t that all rows see, or that some do.
    const int n = (end - begin + kKeys - 1) / kKeys;
    auto run_of = [&](int t) { return window_run(list, begin + kKeys * t); };
    auto next = [&](int t, bool seen_by_all) {
        for (++t; t < n; ++t) {
            const KeyRun run = run_of(t);
            if (run.left <= 0) continue;
            const int keys = min(run.left, kKeys);
            const bool all = kTree ? base >= 0 && run.key + keys <= base
                                   : window_all(a.rule, p_first, p_last, run.key, keys);
            if (all == seen_by_all) break;
        }
        return min(t, n);
    };

    constexpr int kSets = code_sets(D);
    u4 kr[kSets][kLoads], vr[kSets][kLoads];
    // whether the key that this lane looks after is there (none of a tile that was never
    // fetched: behind a walk's last tile the next one is widened all the same, for nobody)
    bool ok[kSets] = {};
    uint32_t ke[kSets], ve[kSets];
    // pages of the rows that the next fetch brings, and of the key looked after
    int page[kLoads + 1];
    // Of the tiles in LDS: the keys that are there, a bit each, what their scores are
    // multiplied by, and the power that their values are relative to.
    uint64_t keys[2];
    float times[2];
    int top[2], most = 0;
    auto row_of = [&](int j) {
        const int f = (int)threadIdx.x + kThreads * j;
        return j == kLoads ? (int)threadIdx.x % kKeys
                           : kEven ? f / kCodes : min(f / kCodes, kKeys - 1);
    };
    auto look = [&](int t) {
        if (t >= n) return;
        const KeyRun run = run_of(t);
#pragma unroll
        for (int j = 0; j <= kLoads; ++j) {
            // (by all threads, of one that is not there the last one's)
            page[j] = table[(run.key + min(row_of(j), run.left - 1)) >> shift];
        }
    };
    auto fetch = [&](int t, auto b) {
        if (t >= n) return;
        constexpr int w = kSets > 1 ? decltype(b)::kIndex : 0;
        const KeyRun run = run_of(t);
        // Row of the cache of a key; of one whose page is none any row.
        auto place = [&](int j) -> int64_t {
            const int its = (unsigned)page[j] < (unsigned)a.few.n_pages ? page[j] : 0;
            return (((int64_t)its * a.few.n_kv + head) << shift) +
                   ((run.key + row_of(j)) & ((1 << shift) - 1));
        };
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int f = (int)threadIdx.x + kThreads * j;
            const int64_t at = place(j) * D + f % kCodes * 16;
            kr[w][j] = *reinterpret_cast<const u4 *>(a.few.k + at);
            vr[w][j] = *reinterpret_cast<const u4 *>(a.few.v + at);
        }
        ok[w] = row_of(kLoads) < run.left && (unsigned)page[kLoads] < (unsigned)a.few.n_pages;
        const int64_t r = place(kLoads);
        ke[w] = a.few.k_exp[r];
        ve[w] = a.few.v_exp[r];
    };
    auto put = [&](int t, auto b, auto seen_by_all) {
        constexpr int w = kSets > 1 ? decltype(b)::kIndex : 0;
        constexpr int at = b.kIndex;
        constexpr bool all = decltype(seen_by_all)::value;
        CodeTile<D> &to = at ? s1 : s0;
        const int mine = ok[w] ? (int)(ke[w] | ve[w] << 16) : -1;  // its powers, or -1
        int key_top = 0;
        keys[at] = __ballot(mine >= 0);  // (of 32 keys: each twice)
        if (all) {
            const uint32_t tops = wave_max2(mine < 0 ? 0 : mine);
            key_top = tops & 255;
            most = max(most, (int)(tops >> 16));
            top[at] = most;
            times[at] = fminf(__builtin_ldexpf(a.few.sl2, key_top - 127), 0x1.fffffep127f);
        } else if (threadIdx.x < kKeys) {
            s_powers[at][threadIdx.x] = ke[w] | ve[w] << 8;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int f = (int)threadIdx.x + kThreads * j, row = f / kCodes;
            const int its = __builtin_amdgcn_ds_bpermute(4 * row, mine);
            if (!kEven && row >= kKeys) continue;
            const int c = f % kCodes, sw = T::swizzle(row & 31);
            // (a value that is left out has to be finite: 0 times it is added)
            if (its < 0) vr[w][j] = u4{0, 0, 0, 0};
            const float kp = power_of(all && its >= 0 ? (its & 255) - key_top : 0);
            const float vp = power_of(all && its >= 0 ? (its >> 16) - most : 0);
            const u2 klo = {kr[w][j][0], kr[w][j][1]}, khi = {kr[w][j][2], kr[w][j][3]};
            const u2 vlo = {vr[w][j][0], vr[w][j][1]}, vhi = {vr[w][j][2], vr[w][j][3]};
            uint8_t *pk = to.k + row * T::kStride, *pv = to.v + row * T::kStride;
            *reinterpret_cast<h8 *>(pk + ((2 * c) ^ sw) * 16) = codes_to<kIn>(klo, kp);
            *reinterpret_cast<h8 *>(pk + ((2 * c + 1) ^ sw) * 16) = codes_to<kIn>(khi, kp);
            *reinterpret_cast<h8 *>(pv + ((2 * c) ^ sw) * 16) = codes_to<kInF16>(vlo, vp);
            *reinterpret_cast<h8 *>(pv + ((2 * c + 1) ^ sw) * 16) = codes_to<kInF16>(vhi, vp);
        }
    };
    // What both kinds of tiles share, from the base-2 scores (times `by`) on; alpha: what
    // the change of the values' power scales the sums by.
    f16v s[kBlocks];
    auto rescale = [&](float mx, int its_top) {
        // (a maximum that has grown by less than 2^6 is not worth the products: the
        // probabilities may as well be 64 times larger, with the same 11 bits)
        const bool grown = mx - m_run > kRaise<kInF16> + 6.f;
        if (__ballot(grown || its_top > ref)) {
            const float m_new = grown ? fmaxf(m_run, lowered<kInF16>(mx)) : m_run;
            float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            l_run *= alpha;
            const int to = max(ref, its_top);
            alpha = __builtin_ldexpf(alpha, ref - to);
            ref = to;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= alpha;
            m_run = m_new;
            large = __ballot(fabsf(m_run) >= kLargeScore && m_run > -INFINITY);
        }
    };
    auto values = [&](const CodeTile<D> &from) {
#pragma unroll
        for (int c = 0; c < 2 * kBlocks; ++c) {
            const h8 p = pack8<kInF16>(s[c >> 1], c & 1);
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                o[d] = mfma32<kInF16>(T::cols32(from.v, 16 * c, 32 * d, lane), p, o[d]);
        }
        products_done();
    };
    auto scores = [&](auto b) {
        const CodeTile<D> &from = b.kIndex ? s1 : s0;
#pragma unroll
        for (int h = 0; h < kBlocks; ++h) s[h] = zero16();
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
#pragma unroll
            for (int h = 0; h < kBlocks; ++h)
                s[h] = mfma32<kIn>(T::rows32(from.k, 32 * h, c, lane), q[c], s[h]);
        }
    };
    auto work = [&](int t, auto b, auto seen_by_all) {
        if (!busy) return;
        constexpr int at = b.kIndex;
        const CodeTile<D> &from = at ? s1 : s0;
        if constexpr (decltype(seen_by_all)::value) {
            float by = times[at];
            const uint64_t all = keys[at];
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
            rescale(mx, top[at]);
            const float m_ref = m_run == -INFINITY ? 0.f : m_run;
            if (large) {  // (see rounded_product)
                const bool its = large >> lane & 1;
#pragma unroll
                for (int e = 0; e < 16 * kBlocks; ++e)
                    s[e >> 4][e & 15] =
                        its ? rounded_product(s[e >> 4][e & 15], by) : s[e >> 4][e & 15];
                by = its ? 1.f : by;
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
        } else {
            const int key0 = run_of(t).key;
            float mx = -INFINITY;
            int its_top = 0;
#pragma unroll
            for (int h = 0; h < kBlocks; ++h) {
                // the keys of the block of 32 that this lane's row sees, a bit each
                uint32_t seen;
                if constexpr (kTree)
                    seen = tree_seen(s_bits[mine], key0 + 32 * h, base);
                else
                    seen = window_bits(a.rule, p_mine, key0 + 32 * h);
                seen = (seen & (uint32_t)(keys[at] >> 32 * h)) >> (4 * (lane >> 5));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const u4 powers = *reinterpret_cast<const u4 *>(
                        &s_powers[at][32 * h + 8 * r + 4 * (lane >> 5)]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool in = seen >> (8 * r + e) & 1;
                        const float x =
                            in ? __builtin_ldexpf(rounded_product(s[h][4 * r + e], a.few.sl2),
                                                  (int)(powers[e] & 255) - 127)
                               : -INFINITY;
                        s[h][4 * r + e] = x;
                        mx = fmaxf(mx, x);
                        its_top = max(its_top, in ? (int)(powers[e] >> 8) : 0);
                    }
                }
            }
            mx = max_xor32(mx);
            const auto both = __builtin_amdgcn_permlane32_swap(its_top, its_top, false, false);
            rescale(mx, max((int)both[0], (int)both[1]));
            const float m_ref = m_run == -INFINITY ? 0.f : m_run;
            float sum = 0.f;
#pragma unroll
            for (int h = 0; h < kBlocks; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // (all of a tile's powers at once would spill at d = 64)
                    if (r % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                    const u4 powers = *reinterpret_cast<const u4 *>(
                        &s_powers[at][32 * h + 8 * r + 4 * (lane >> 5)]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = __builtin_amdgcn_exp2f(s[h][4 * r + e] - m_ref);
                        sum += x;
                        // (of a key that it does not see: 0, whatever its power)
                        s[h][4 * r + e] =
                            __builtin_ldexpf(x, (int)(powers[e] >> 8) - ref);
                    }
                }
            l_run += sum;
        }
        values(from);
    };
    auto walk = [&](auto all) {
        // tiles: in LDS, waiting in registers, to be fetched, to be looked up
        int id[kSets + 3];
        id[0] = next(-1, all.value);
        if (id[0] >= n) return;
#pragma unroll
        for (int k = 1; k < kSets + 3; ++k) id[k] = next(id[k - 1], all.value);
        auto step = [&](auto here, auto other) {
            __syncthreads();  // tile id[0] is there, and nobody reads the other buffer
            scores(here);
            put(id[1], other, all);
            fetch(id[1 + kSets], other);
            look(id[2 + kSets]);
            work(id[0], here, all);
#pragma unroll
            for (int k = 0; k < kSets + 2; ++k) id[k] = id[k + 1];
            id[kSets + 2] = next(id[kSets + 1], all.value);
        };
        look(id[0]);
        fetch(id[0], Buffer<0>());
        look(id[1]);
        if (kSets > 1) {
            fetch(id[1], Buffer<1>());
            look(id[2]);
        }
        __syncthreads();  // nobody reads the buffers any more
        put(id[0], Buffer<0>(), all);
        fetch(id[kSets], Buffer<0>());
        look(id[kSets + 1]);
        while (id[0] < n) {
            step(Buffer<0>(), Buffer<1>());
            if (id[0] < n) step(Buffer<1>(), Buffer<0>());
        }
    };
    walk(std::true_type());
    walk(std::false_type());

    const float l = __builtin_ldexpf(sum_xor32(l_run), -kRaise<kInF16>);
    // (two waves to a buffer where there are eight)
    constexpr int kOwn = T::kBytes * 4 / W;
    const int part4 = wave & 3;
    uint8_t *const lds =
        (part4 == 0 ? s0.k : part4 == 1 ? s0.v : part4 == 2 ? s1.k : s1.v) + wave / 4 * kOwn;
    __syncthreads();  // nobody reads the tiles
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int k = 0; k < 16; ++k)
            o[d][k] = __builtin_ldexpf(o[d][k], ref - 127 - kRaise<kInF16>);
    if (!a.direct) {
        const int64_t part = part0 + 32 * wave;
        store_part32<D, kOwn / 128 / 32 * 32>(lds, o, 1.f, a.few.part_o + part * D, D,
                                                   rows - 32 * wave, lane);
        if (there && lane < 32) {
            a.few.part_ml[2 * (part + lane)] = m_run;
            a.few.part_ml[2 * (part + lane) + 1] = l;
        }
        return;
    }
    auto at = [&](int r) { return query_row(a.few.q, head, row0 + 32 * wave + r); };
    store_rows32<D, kIn, D>(lds, o, l == 0.f ? 0.f : 1.f / l, a.few.O, at, rows - 32 * wave, 0,
                            lane);
    if (there && lane < 32) a.few.lse[at(lane)] = natural_lse(m_run + kRaise<kInF16>, l);
}

template <int D, int kIn, int kMask>
void launch_attend_own_d(const AttendArgs &a, int64_t grid, hipStream_t s)
{
    if constexpr (own_wide(D)) {
        if (a.own_rows == 2 * kManyRows) {
            k_attend_own<D, kIn, kMask, 8><<<(unsigned)grid, 512, 0, s>>>(a);
            return;
        }
    }
    k_attend_own<D, kIn, kMask, 4><<<(unsigned)grid, 256, 0, s>>>(a);
}

template <int D, int kIn>
hipError_t launch_attend_window_d(const AttendArgs &a, hipStream_t s)
{
    const int64_t grid = (int64_t)a.n_seqs * a.splits * a.few.n_kv * a.row_blocks;
    if (a.own_rows > kFewRows)
        launch_attend_own_d<D, kIn, kWindowMask>(a, grid, s);
    else
        k_attend_window<D, kIn><<<(unsigned)grid, 64 * kFewWaves, 0, s>>>(a);
    launch_attend_join_d<D, kIn>(a, s);
    return hipGetLastError();
}

template <int D, int kIn>
hipError_t launch_attend_tree_d(const AttendArgs &a, hipStream_t s)
{
    const int64_t own = (int64_t)a.own_items * a.few.n_kv * a.row_blocks;
    const int64_t prefix = (int64_t)a.prefix_splits * a.few.n_kv * a.prefix_blocks;
    if (a.own_rows > kFewRows) {
        // (the prefix by one kernel or the other)
        if (prefix && !a.prefix_many)
            k_attend_tree<D, kIn><<<(unsigned)prefix, 64 * kFewWaves, 0, s>>>(a);
        launch_attend_own_d<D, kIn, kTreeMask>(a, own + (a.prefix_many ? prefix : 0), s);
    } else {
        if (a.prefix_many) {
            const hipError_t e = launch_attend_prefix_d<D, kIn>(a, s);
            if (e != hipSuccess) return e;
        }
        k_attend_tree<D, kIn>
            <<<(unsigned)(own + (a.prefix_many ? 0 : prefix)), 64 * kFewWaves, 0, s>>>(a);
    }
    launch_attend_join_d<D, kIn>(a, s);
    return hipGetLastError();
}

hipError_t launch_attend_window_f16(const AttendArgs &a, int d, hipStream_t s);
hipError_t launch_attend_window_bf16(const AttendArgs &a, int d, hipStream_t s);
hipError_t launch_attend_tree_f16(const AttendArgs &a, int d, hipStream_t s);
hipError_t launch_attend_tree_bf16(const AttendArgs &a, int d, hipStream_t s);

}  // namespace f3s
