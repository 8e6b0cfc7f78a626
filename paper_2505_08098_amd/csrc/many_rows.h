// Attention of many query rows to a range of keys: forward of cross attention
// (f3s_cross_forward).
//
// A workgroup of four waves has up to 128 query rows, 32 to a wave, and walks
// the keys in tiles of 64 (d > 128: 32) that all four use: K and V tiles pass
// through LDS in two buffers, the next one filled while the last is worked on,
// with one barrier a tile.  With 128 rows a tile of K and V (4 d bytes a key) feeds
// 512 d operations a key: the matrix units and the softmax's vector
// instructions are the bound, not memory.
//
// S^T = K Q^T with the 32x32x16 product: a lane holds one query row and half
// of a tile's keys, which is at once the operand layout of O^T += V^T P^T (V
// read transposed from LDS), so the probabilities never leave their lane.  The
// running maximum needs one exchange a tile, between the two halves of a wave;
// sums stay in the lane until the end.
//
// 2 x 4,050 tokens, 32 heads of 128 over 8, 8,100 keys, bf16: 1,060 us, 1,010
// TFLOP/s, where a library's product of 8,192^3 reaches 1,200 to 1,320 by card.  The
// clock falls to 1.9 GHz, the matrix units are busy 48% of its cycles and the vector unit as
// long again; more waves or earlier reads gained nothing, LDS reads without bank conflicts
// 2%.  Power seems to be the bound.
//
// P enters the value product in the inputs' type: rounded to nearest, a bf16 result
// is off by 0.0023 of its size instead of the 0.0017 of its own rounding (fp16 0.0003
// and 0.0002).  Two 16-bit terms of P would take half as many products again.
#pragma once

#include <type_traits>

#include "few_rows.h"

namespace f3s {

constexpr int kManyRows = 128;  // query rows of a workgroup
constexpr int kManyThreads = 256;
// Rows of the other side in a tile (wide rows: fewer, or the registers that
// hold the next tile on its way into LDS would spill).
constexpr int many_keys(int d) { return d <= 128 ? 64 : 32; }

// D(32x32, fp32) += A(32x16) B(16x32), f16 or bf16.  Lane l holds A row l % 32
// and B column l % 32 with reduction slots 8 (l / 32) .. + 7, and of D column
// l % 32 the rows 8 (r / 4) + 4 (l / 32) + r % 4, r = 0 .. 15 (checked on the GPU).
template <int kIn>
__device__ __forceinline__ f16v mfma32(h8 a, h8 b, f16v c)
{
    if constexpr (kIn == kInBF16) {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a),
                                                       __builtin_bit_cast(b8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
}

__device__ __forceinline__ f16v zero16()
{
    f16v z;
#pragma unroll
    for (int k = 0; k < 16; ++k) z[k] = 0.f;
    return z;
}

// A tile of one head's rows in LDS, and how it gets there.
//
// d a power of two: the loads write LDS themselves (16 bytes a lane), which
// takes no registers.  A wave's load fills 1 KB in lane order, so rows cannot be
// padded; instead the 16-byte pieces of a row change places, piece p of row r
// standing at p ^ swizzle(r).  The rows that share banks (16 / pieces rows stand in 256
// bytes) differ in it by the piece's upper bits first, then by its lower ones: so the 16
// rows of a plain operand read (rows32) meet different banks, and so do the 4 rows of
// four neighbouring pieces of a transposed one (cols32), and so do those that store every
// other piece of neighbouring rows (attend_many.h).  A swizzle that moved
// neighbouring rows apart by two pieces made the latter meet each bank twice (two
// sequences of 8,100 tokens, window 1,024, 16 heads of 128 over 4: 792 us a training step
// instead of 713; 2 x 4,050 tokens over 8,100 keys, 32 heads over 8: 1,080 us instead of
// 1,060).
// Other d: through registers, into padded rows.
template <int D, int R = many_keys(D)>
struct ManyTile {
    static constexpr bool kDirect = (D & (D - 1)) == 0;
    static constexpr int kRows = R;
    static constexpr int kPieces = D / 8;              // 16-byte pieces of a row
    static constexpr int kStride = 2 * D + (kDirect ? 0 : 32);  // bytes
    static constexpr int kBytes = kRows * kStride;
    static constexpr int kLoads = (kRows * kPieces + kManyThreads - 1) / kManyThreads;
    static constexpr bool kEven = kRows * kPieces % kManyThreads == 0;
    static_assert(!kDirect || kEven, "");

    static __device__ __forceinline__ int swizzle(int row)
    {
        if constexpr (!kDirect) return 0;
        // (256 bytes are all banks, which 16 / kPieces rows of short ones share)
        if constexpr (kPieces >= 16) return (row & 3) << 2 | ((row >> 2 & 3) ^ (row & 1));
        if constexpr (kPieces == 8) return (row >> 1 & 1) << 2 | ((row >> 2 & 3) ^ (row >> 1 & 1));
        return row >> 2 & 3;
    }

    u4 r[kDirect ? 1 : kLoads];

    // Start bringing in the rows that stand offset(0 .. kRows - 1) bytes (below
    // 2^32) behind base, which is the same for all lanes: into the tile (kDirect:
    // it is there after settle() of every wave and a barrier), or into registers
    // for put().
    template <typename F>
    __device__ __forceinline__ void fetch(uint8_t *tile, const uint8_t *base, F offset)
    {
        if constexpr (kDirect) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int f = (int)threadIdx.x + kManyThreads * j, row = f / kPieces;
                const int piece = f % kPieces ^ swizzle(row);
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)(base + (offset(row) + piece * 16)),
                    (__attribute__((address_space(3))) void *)(tile + 1024 * wave + 4096 * j),
                    16, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int f = (int)threadIdx.x + kManyThreads * j;
                const int row = kEven ? f / kPieces : min(f / kPieces, kRows - 1);
                r[j] = *reinterpret_cast<const u4 *>(base + (offset(row) + f % kPieces * 16));
            }
        }
    }
    __device__ __forceinline__ void put(uint8_t *tile)
    {
        if constexpr (!kDirect) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int f = (int)threadIdx.x + kManyThreads * j, row = f / kPieces;
                if (kEven || row < kRows)
                    *reinterpret_cast<u4 *>(tile + row * kStride + f % kPieces * 16) = r[j];
            }
        }
    }
    // Operand with the tile's rows row .. row + 31 and elements 16 c .. + 15
    // (row a multiple of 32).
    static __device__ __forceinline__ h8 rows32(const uint8_t *tile, int row, int c, int lane)
    {
        const int i = lane & 31;
        const int at = (row + i) * kStride + ((2 * c + (lane >> 5)) ^ swizzle(i)) * 16;
        return *reinterpret_cast<const h8 *>(tile + at);
    }
    // Operand with elements d .. d + 31 as rows and the tile's rows row .. + 15 as
    // reduction slots (d a multiple of 32, row of 16), in the order in which a lane
    // holds them of an S^T accumulator: 4 h + 0..3 and 8 + 4 h + 0..3 (h: the
    // lane's half).
    static __device__ __forceinline__ h8 cols32(const uint8_t *tile, int row, int d, int lane)
    {
        const int s = lane & 15, i = 4 * (lane >> 5) + (s >> 2);
        const int piece = d / 8 + 2 * (lane >> 4 & 1) + (s >> 1 & 1);
        // (one sum each, not a chain: behind five steps from a variable the compiler
        // no longer tells it from the other buffer, and waits for the loads into that)
        const int lo = (row + i) * kStride + (piece ^ swizzle(row % 32 + i)) * 16 + 8 * (s & 1);
        const int hi =
            (row + i + 8) * kStride + (piece ^ swizzle(row % 32 + i + 8)) * 16 + 8 * (s & 1);
        return cat44(lds_read_tr(reinterpret_cast<const _Float16 *>(tile + lo)),
                     lds_read_tr(reinterpret_cast<const _Float16 *>(tile + hi)));
    }
};

// This wave's direct loads have arrived (vmcnt(0); the compiler does not wait for
// loads that write LDS by itself).
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// The walk over n tiles, in two buffers: fetch(t, b) starts tile t on its way
// into buffer b, put(t, b) takes there what waits in registers, work(t, b) uses
// it.  While a tile is worked on the next one arrives.  The buffer is a type
// (Buffer<0>, Buffer<1>) and each has LDS variables of its own: where they were
// one array, the compiler held a transposed read to depend on the loads into
// the other half and waited for them (dK and dV of pairs of 4,050, 16 heads of
// 128 over 4: 700 us instead of 726).
template <int B>
struct Buffer {
    static constexpr int kIndex = B;
};
template <bool kDirect, typename Fetch, typename Put, typename Work>
__device__ __forceinline__ void walk_tiles(int n, Fetch fetch, Put put, Work work)
{
    auto step = [&](int t, auto here, auto there) {
        if constexpr (kDirect) settle();
        __syncthreads();  // tile t is there, and nobody reads the other buffer
        const bool more = t + 1 < n;
        if constexpr (kDirect) {
            if (more) fetch(t + 1, there);
            work(t, here);
            if (more) put(t + 1, there);
        } else {
            if (more) {
                put(t + 1, there);
                fetch(min(t + 2, n - 1), here);
            }
            work(t, here);
        }
    };
    if (n > 0) {
        fetch(0, Buffer<0>());
        put(0, Buffer<0>());
        if constexpr (!kDirect) fetch(n > 1 ? 1 : 0, Buffer<1>());
    }
    for (int t = 0; t < n; t += 2) {
        step(t, Buffer<0>(), Buffer<1>());
        if (t + 1 < n) step(t + 1, Buffer<1>(), Buffer<0>());
    }
}

// 32 rows of one head as an operand (row row + lane % 32; zeros from `rows` on).
template <int D>
__device__ __forceinline__ void load_rows32(h8 (&x)[D / 16], const void *src, int64_t at,
                                            bool there, uint32_t flip, int lane)
{
    const _Float16 *p = reinterpret_cast<const _Float16 *>(src) + at * D + 8 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u4 v = *reinterpret_cast<const u4 *>(p + 16 * c);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = there ? v[k] ^ flip : 0u;
        x[c] = __builtin_bit_cast(h8, v);
    }
}

// Eight of an accumulator's values as an operand of 16 reduction slots.
template <int kIn>
__device__ __forceinline__ h8 pack8(const f16v &x, int half)
{
    h8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = to16<kIn>(x[8 * half + e]);
    return p;
}

__device__ __forceinline__ float sum_xor32(float v)
{
    const int b = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}

// Stores a wave's 32 result rows of kCols columns from an O^T-like accumulator,
// scaled and rounded: `rows` of them, row r as row at(r) of `to` from column
// `col` on.  A lane holds 8 bytes here and there of one row; through 64 kCols
// bytes of LDS (the wave's own, nothing else in it in use) they become whole
// rows of 16-byte pieces (dK and dV of 56 sequences of 11 to 22 tokens over 964 to
// 2,891, 16 heads of 128 over 4: 131 us instead of 175).
template <int D, int kIn, int kCols, typename At>
__device__ __forceinline__ void store_rows32(uint8_t *lds, const f16v (&x)[kCols / 32],
                                             float scale, void *to, At at, int rows, int col,
                                             int lane)
{
    constexpr int kPieces = kCols / 8, kMask = kPieces % 8 ? 3 : 7;
    asm("" : "+v"(lane));  // (what follows from it is not kept in registers until here)
    const int i = lane & 31;
#pragma unroll
    for (int d = 0; d < kCols / 32; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            h4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = to16<kIn>(x[d][4 * k + e] * scale);
            *reinterpret_cast<h4 *>(lds + i * (2 * kCols) + ((4 * d + k) ^ (i & kMask)) * 16 +
                                    8 * (lane >> 5)) = v;
        }
    tile_fence<kFewWaves>();
#pragma unroll
    for (int j = 0; j < kPieces / 2; ++j) {
        const int f = lane + 64 * j, row = f / kPieces, piece = f % kPieces;
        if (row < rows)
            *reinterpret_cast<u4 *>(reinterpret_cast<uint8_t *>(to) +
                                    (at(row) * D + col) * 2 + piece * 16) =
                *reinterpret_cast<const u4 *>(lds + row * (2 * kCols) +
                                              (piece ^ (row & kMask)) * 16);
    }
    tile_fence<kFewWaves>();
}

// The same into partial sums: fp32, row r at part + r * stride, kChunk columns at
// a time through 128 kChunk bytes of LDS (the prefix of attend_many.h: 54.2 us
// instead of 55.7).
template <int kCols, int kChunk>
__device__ __forceinline__ void store_part32(uint8_t *lds, const f16v (&x)[kCols / 32],
                                             float scale, float *part, int stride, int rows,
                                             int lane)
{
    asm("" : "+v"(lane));
    const int i = lane & 31;
#pragma unroll
    for (int first = 0; first < kCols; first += kChunk) {
        const int cols = kCols - first < kChunk ? kCols - first : kChunk, pieces = cols / 4;
#pragma unroll
        for (int d = 0; d < cols / 32; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f16v &y = x[first / 32 + d];
                *reinterpret_cast<f4 *>(lds + i * (4 * cols) +
                                        ((8 * d + 2 * k + (lane >> 5)) ^ (i & 7)) * 16) =
                    f4{y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]} * scale;
            }
        tile_fence<kFewWaves>();
#pragma unroll
        for (int j = 0; j < pieces / 2; ++j) {
            const int f = lane + 64 * j, row = f / pieces, piece = f % pieces;
            if (row < rows)
                *reinterpret_cast<u4 *>(part + (int64_t)row * stride + first + 4 * piece) =
                    *reinterpret_cast<const u4 *>(lds + row * (4 * cols) +
                                                  (piece ^ (row & 7)) * 16);
        }
        tile_fence<kFewWaves>();
    }
}

// What many_rows, and the dQ pass of cross_backward.h, ask of an item of either kind.
//
// The positions of a wave's tokens: the first's, the last's and this lane's (none
// where all keys are seen).
struct RowPositions {
    int32_t first, last, mine;
};
__device__ __forceinline__ RowPositions row_positions(const QueryRows &, const DenseItem &, int,
                                                      int)
{
    return {};
}
__device__ __forceinline__ RowPositions row_positions(const QueryRows &q, const WindowItem &it,
                                                      int wave, int mine)
{
    const int last = min(32 * wave + 31, it.rows - 1);
    return {(int)row_token(q, it.row + 32 * wave) + it.shift,
            (int)row_token(q, it.row + last) + it.shift,
            (int)row_token(q, it.row + mine) + it.shift};
}
// The row of K that key 0 is, and the keys from place t of the walk on.
__device__ __forceinline__ int32_t key_base(const DenseItem &it) { return it.other; }
__device__ __forceinline__ int32_t key_base(const WindowItem &it) { return it.key0; }
__device__ __forceinline__ KeyRun key_run(const DenseItem &it, int t)
{
    return {t, it.others - t};
}
__device__ __forceinline__ KeyRun key_run(const WindowItem &it, int t)
{
    return window_run(it.keys, it.other + t);
}

// Masks of an accumulator by bits: of 32 rows a lane holds 16, and of its bits it takes
// those.  Element e stands at bit 8 (e / 4) + e % 4 of what is left: two instructions an
// element (one bit widened to a word, a select by its bits).
__device__ __forceinline__ uint32_t lane_bits(uint32_t bits, int lane)
{
    return bits >> (4 * (lane >> 5));
}
__device__ __forceinline__ uint32_t element_mask(uint32_t bits, int e)
{
    return (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (e >> 2) + (e & 3), 1);
}
__device__ __forceinline__ float kept_score(float x, uint32_t bits, int e)  // or -inf
{
    return masked_score(x, element_mask(bits, e));
}
__device__ __forceinline__ float kept_value(float x, uint32_t bits, int e)  // or 0
{
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & element_mask(bits, e));
}

// Waves per SIMD that the registers leave room for.
constexpr int many_waves(int d) { return d <= 64 ? 3 : d <= 128 ? 2 : 1; }

// Item: DenseItem (rows see all keys of their range) or WindowItem.
template <int D, int kIn, typename Item>
__device__ __forceinline__ void many_rows(const FewArgs &a, const Item &it, const WindowRule &rule)
{
    constexpr bool kWindow = std::is_same<Item, WindowItem>::value;
    using T = ManyTile<D>;
    constexpr int kKeys = T::kRows, kBlocks = kKeys / 32;
    __shared__ __attribute__((aligned(16))) uint8_t s_k0[T::kBytes], s_k1[T::kBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_v0[T::kBytes], s_v1[T::kBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = 32 * wave + (lane & 31);  // this lane's query row
    const bool there = mine < it.rows;
    const bool busy = 32 * wave < it.rows;     // (the wave has rows at all)
    const RowPositions at_p = row_positions(a.q, it, wave, there ? mine : 0);

    h8 q[D / 16];
    load_rows32<D>(q, a.Q, query_row(a.q, it.head, (int64_t)it.row + (there ? mine : 0)), there,
                   a.flip, lane);
    f16v o[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = zero16();
    float m_run = -INFINITY, l_run = 0.f;  // maximum, lowered by kRaise
    uint64_t large = 0;  // lanes where it is from kLargeScore on

    T tk, tv;
    const uint32_t row_bytes = (uint32_t)a.n_kv * (2 * D);
    const uint64_t base = (uint64_t)key_base(it) * row_bytes + (uint32_t)it.head * (2 * D);
    const uint8_t *const K = reinterpret_cast<const uint8_t *>(a.K) + base;
    const uint8_t *const V = reinterpret_cast<const uint8_t *>(a.V) + base;
    auto fetch = [&](int t, auto b) {
        // rows behind the range: its last one again (whatever stands there may
        // not be finite, and 0 times it is added)
        const KeyRun run = key_run(it, kKeys * t);
        const int first = run.key, last = kWindow ? max(run.left - 1, 0) : run.left - 1;
        const uint64_t at = (uint64_t)first * row_bytes;
        auto offset = [&](int row) { return (uint32_t)min(row, last) * row_bytes; };
        tk.fetch(b.kIndex ? s_k1 : s_k0, K + at, offset);
        tv.fetch(b.kIndex ? s_v1 : s_v0, V + at, offset);
    };
    auto put = [&](int, auto b) {
        tk.put(b.kIndex ? s_k1 : s_k0);
        tv.put(b.kIndex ? s_v1 : s_v0);
    };
    auto work = [&](int t, auto b) {
        if (!busy) return;
        const KeyRun run = key_run(it, kKeys * t);
        const int left = run.left;
        if (kWindow &&
            (left <= 0 || window_none(rule, at_p.first, at_p.last, run.key, min(left, kKeys))))
            return;
        const uint8_t *k = b.kIndex ? s_k1 : s_k0, *v = b.kIndex ? s_v1 : s_v0;
        f16v s[kBlocks];
#pragma unroll
        for (int h = 0; h < kBlocks; ++h) s[h] = zero16();
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
#pragma unroll
            for (int h = 0; h < kBlocks; ++h)
                s[h] = mfma32<kIn>(T::rows32(k, 32 * h, c, lane), q[c], s[h]);
        }
        if constexpr (kWindow) {
            if (left < kKeys || !window_all(rule, at_p.first, at_p.last, run.key, kKeys)) {
#pragma unroll
                for (int h = 0; h < kBlocks; ++h) {
                    const uint32_t bits =
                        lane_bits(window_bits(rule, at_p.mine, run.key + 32 * h) &
                                      bits_to(left - 32 * h - 1),
                                  lane);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[h][e] = kept_score(s[h][e], bits, e);
                }
            }
        } else if (left < kKeys) {
#pragma unroll
            for (int e = 0; e < 16 * kBlocks; ++e) {
                const int key = 32 * (e >> 4) + 8 * ((e & 15) >> 2) + 4 * (lane >> 5) + (e & 3);
                if (key >= left) s[e >> 4][e & 15] = -INFINITY;
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < 16 * kBlocks; ++e) mx = fmaxf(mx, s[e >> 4][e & 15]);
        mx = rounded_product(max_xor32(mx), a.sl2);
        // (a maximum that has grown by less than 2^6 is not worth the products: the
        // probabilities may as well be 64 times larger, with the same bits)
        const bool grown = mx - m_run > kRaise<kIn> + 6.f;
        if (__ballot(grown)) {
            // (a window's rows that see other keys do not change a row's bits)
            const float m_new = kWindow && !grown ? m_run : fmaxf(m_run, lowered<kIn>(mx));
            const float alpha =
                __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            l_run *= alpha;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= alpha;
            m_run = m_new;
            large = __ballot(fabsf(m_run) >= kLargeScore);
        }
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;
        float by = a.sl2;
        if (large) {  // (see rounded_product)
            const bool its = !kWindow || (large >> lane & 1);
#pragma unroll
            for (int e = 0; e < 16 * kBlocks; ++e)
                s[e >> 4][e & 15] =
                    its ? rounded_product(s[e >> 4][e & 15], by) : s[e >> 4][e & 15];
            by = its ? 1.f : by;
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16 * kBlocks; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], by, -m_ref));
            s[e >> 4][e & 15] = p;
            sum += p;
        }
        l_run += sum;
#pragma unroll
        for (int c = 0; c < 2 * kBlocks; ++c) {
            const h8 p = pack8<kIn>(s[c >> 1], c & 1);
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                o[d] = mfma32<kIn>(T::cols32(v, 16 * c, 32 * d, lane), p, o[d]);
        }
        products_done();
    };
    walk_tiles<T::kDirect>((it.others + kKeys - 1) / kKeys, fetch, put, work);
    constexpr float kLower = 1.f / (1 << kRaise<kIn>);
    const float l = sum_xor32(l_run) * kLower;
    const int col = 4 * (lane >> 5);
    uint8_t *const lds = wave == 0 ? s_k0 : wave == 1 ? s_k1 : wave == 2 ? s_v0 : s_v1;
    __syncthreads();  // nobody reads the tiles
    if (it.part >= 0) {
        store_part32<D, T::kBytes / 128 / 32 * 32>(
            lds, o, kLower, a.part_o + ((int64_t)it.part + 32 * wave) * D, D, it.rows - 32 * wave,
            lane);
        if (there && col == 0) {
            a.part_ml[2 * ((int64_t)it.part + mine)] = m_run;
            a.part_ml[2 * ((int64_t)it.part + mine) + 1] = l;
        }
        return;
    }
    auto at = [&](int r) { return query_row(a.q, it.head, (int64_t)it.row + 32 * wave + r); };
    store_rows32<D, kIn, D>(lds, o, l == 0.f ? 0.f : kLower / l, a.O, at, it.rows - 32 * wave, 0,
                            lane);
    if (there && col == 0) a.lse[at(lane & 31)] = natural_lse(m_run + kRaise<kIn>, l);
}

template <int D, int kIn>
__global__ __launch_bounds__(kManyThreads, many_waves(D)) void k_cross_many(
    FewArgs a, const DenseItem *items)
{
    const DenseItem it = items[blockIdx.x];
    many_rows<D, kIn>(a, it, {});
}

template <int D, int kIn>
hipError_t launch_cross_many_d(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s)
{
    if (p.n_fwd) k_cross_many<D, kIn><<<p.n_fwd, kManyThreads, 0, s>>>(a, p.fwd);
    return hipGetLastError();
}

hipError_t launch_cross_many_f16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s);
hipError_t launch_cross_many_bf16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s);

}  // namespace f3s
