/*
 * f3s_cache.h -- keys and values of generated tokens in a paged cache of 8
 * bits per value, and the attention that reads it (libf3s.so).
 *
 * A row (the d values of one token and one key head) is stored as d codes of
 * the OCP 8-bit float e4m3 and one byte that holds a power of two: value =
 * code * 2^(byte - 127), with the smallest power that keeps the row's largest
 * magnitude at or below 448, e4m3's largest (at least 2^-127).  Codes are
 * rounded to the nearest, to the even one in the middle.  A power of two adds
 * no rounding of its own.  (A value next to its type's largest may be
 * rounded up beyond it and then reads back as infinity: f16 above 63488, bf16
 * above 2^128 - 2^124.)  NaN and infinite elements are stored as NaN and do
 * not count for the power.
 *
 * Pages: page p holds page_size tokens of every key head.  A sequence's
 * positions 0, 1, ... lie in the pages that its row of the table names, in
 * order.  An entry outside [0, n_pages) is no page: rows that would lie there
 * are not written, read back as zeros and do not take part in attention.
 *
 * Lengths live on the device and may change between calls (or between the
 * replays of a captured graph): lens[b] is the sequence's number of tokens
 * INCLUDING the n_new newest, at the positions lens[b] - n_new + t for t = 0
 * .. n_new - 1.  A t with a negative position is padding (sequences shorter
 * than n_new, whose rows then stand at the end: padded on the left).
 * Negative lengths count as 0; positions behind the table are left out.
 */
#ifndef F3S_CACHE_H
#define F3S_CACHE_H

#include "f3s.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void *k, *v;             /* device, codes [n_pages, n_kv_heads, page_size, d],
                                16-byte aligned                                   */
    uint8_t *k_exp, *v_exp;  /* device, powers [n_pages, n_kv_heads, page_size],
                                16-byte aligned                                   */
    int32_t n_pages;         /* >= 1                                              */
    int32_t n_kv_heads;      /* >= 1                                              */
    int32_t page_size;       /* 16, 32, 64, 128 or 256                            */
    int32_t d;               /* multiple of 32, 32 <= d <= 256                    */
} f3s_cache_t;

/*
 * Write the n_new newest rows of every sequence.
 *   K, V       device, dtype (F3S_DTYPE_F16 or F3S_DTYPE_BF16), [n_seqs, n_new,
 *              n_kv_heads, d] row-major, 16-byte aligned
 *   table      device int32 [n_seqs, max_pages]
 *   lens       device int32 [n_seqs], the lengths after this call
 * Two rows of one call must not lie at the same place (a page named twice):
 * what such a place then holds is not defined.  K and V must not overlap the
 * cache, nor its four parts each other, but that one place for keys and values takes
 * the same rows as K and V (a cache that is only read may be laid out in any way).
 * F3S_ERR_TOO_LARGE from 2^27 rows on (sequences, tokens, key heads; from 2^28 up
 * to d = 128, 2^29 up to 64, 2^30 at 32).
 * Asynchronous on `stream`; no allocation, no synchronisation.
 */
f3s_status_t f3s_cache_write(const f3s_cache_t *cache, const void *K, const void *V,
                             f3s_dtype_t dtype, const int32_t *table, int32_t max_pages,
                             const int32_t *lens, int32_t n_seqs, int32_t n_new,
                             hipStream_t stream);

/*
 * Read the n_new newest rows of every sequence back: K, V (laid out as for
 * f3s_cache_write) receive the values rounded to dtype (F16, BF16 or F32) to
 * nearest even, zeros where a row has no place.  K or V may be NULL; they must
 * not overlap each other or anything that is read.
 */
f3s_status_t f3s_cache_read(const f3s_cache_t *cache, void *K, void *V, f3s_dtype_t dtype,
                            const int32_t *table, int32_t max_pages, const int32_t *lens,
                            int32_t n_seqs, int32_t n_new, hipStream_t stream);

/*
 * Keep some of the n_new newest tokens of every sequence (those of a draft that were
 * accepted) and drop the others: the rows of the kept tokens move to the front of the
 * n_new, in order.
 *   picks      device int32 [n_seqs, n_picks]: the kept tokens t of 0 .. n_new - 1,
 *              ascending.  The first entry that is not larger than the one before it, is
 *              outside 0 .. n_new - 1 or names a padding row (a negative position) ends
 *              the list (-1, say)
 *   new_lens   device int32 [n_seqs]: the lengths after this call, max(lens[b] - n_new, 0)
 *              plus the number of tokens kept
 * table and lens as above.  A row that has no place (its page is none) is not moved, and
 * nothing is moved onto one.  The places behind the new length hold what they held or
 * what was moved away.  Every page of the n_new tokens belongs to one sequence.  The
 * cache's four parts must not share memory with each other or with the other arguments,
 * nor new_lens with any of them.  F3S_ERR_TOO_LARGE beyond 2^30 picks of a sequence.
 * Asynchronous on `stream`; no allocation, no synchronisation; deterministic.
 */
f3s_status_t f3s_cache_keep(const f3s_cache_t *cache, const int32_t *table, int32_t max_pages,
                            const int32_t *lens, int32_t n_seqs, int32_t n_new,
                            const int32_t *picks, int32_t n_picks, int32_t *new_lens,
                            hipStream_t stream);

/*
 * Attention of the n_new newest tokens of every sequence to a prefix that all
 * sequences share and to their own cached keys.  Token t sees the whole
 * prefix and its own positions up to lens[b] - n_new + t (itself, if it was
 * written).  Query head h uses key head h / (n_heads / n_kv_heads).
 *
 *     O = softmax(scale Q K^T) V over the keys that the token sees
 *
 *   Q, O       device, dtype (F16 or BF16), [n_seqs, n_new, n_heads, d]
 *              row-major, 16-byte aligned; O must not overlap an input
 *   lse        device fp32 [n_seqs, n_new, n_heads]: log of the sum of the
 *              exponentials (-inf, and O = 0, for a token that sees no key)
 *   table, lens  as above; keys behind the table do not take part, and it has
 *              room for 2^30 tokens at most
 *   prefix     device int32 [ceil(prefix_len / page_size)]: the pages of the
 *              prefix (its last one may end inside); NULL if prefix_len is 0;
 *              prefix_len <= 2^30
 *   scale      finite
 *   workspace  device, at least f3s_cache_attend_workspace_bytes(...) bytes,
 *              256-byte aligned; needs no initialisation, must not overlap
 *              anything else of the call, and calls that overlap in time need
 *              one each.  NULL if that is 0
 * Inputs must be finite, and so must every row below a sequence's length: one that
 * is not may reach all of its tokens, those before it too.  Scores, sums and statistics are fp32 (products of Q with
 * codes, before and after scaling, and |V| times the number of keys have to stay
 * below 2^127); the products with V are f16, relative to the largest power of two
 * among the values that the token has seen so far: beside 2^-11 of its probability
 * a key adds an error of up to 2^-33 of the largest |value| that the token sees.
 * The work is divided on the device, by the lengths that it finds there: a captured
 * call stays right when they change.  A prefix is read once for many sequences: for
 * 16 query rows of a key head at a time, or, with many rows and much work, for 128
 * (environment F3S_PREFIX_ROWS=16 or 128 forces one).  Deterministic.
 * Asynchronous on `stream`; no allocation, no synchronisation.
 */
f3s_status_t f3s_cache_attend(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                              void *O, float *lse, const int32_t *table, int32_t max_pages,
                              const int32_t *lens, int32_t n_seqs, int32_t n_new,
                              int32_t n_heads, const int32_t *prefix, int32_t prefix_len,
                              float scale, void *workspace, size_t workspace_bytes,
                              hipStream_t stream);

/* Device bytes of scratch such a call needs (0 also for sizes that it refuses).
   Host-only. */
size_t f3s_cache_attend_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                        int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                        int32_t prefix_len);

/*
 * The same without a prefix and with a window: a token at position p sees its own
 * sequence's positions j <= p with p - j < window (itself, if it was written, and the
 * window - 1 before it) or j < sinks.  A token that sees no key gives O = 0, lse = -inf.
 *   window, sinks   >= 0; from 2^30 on as 2^30
 *   workspace       at least f3s_cache_attend_window_workspace_bytes(...) bytes
 * Query rows of a sequence and key head (n_new times n_heads / n_kv_heads) are worked on 16
 * at a time, or 128 or 256 where they are many (environment F3S_OWN_ROWS=16, 128 or, for d
 * of 96 and 128, 256 forces one; read by every call, that for the workspace's size too).  In
 * the latter two, keys that all of these rows see have their powers of two applied relative
 * to the largest of their tile (K) or among the keys before (V), f16: beside what
 * f3s_cache_attend says a key 2^15 times smaller than that has its score's part off by 2^-25
 * of the largest.  What a token does not see changes no bit of its result.
 */
f3s_status_t f3s_cache_attend_window(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                                     void *O, float *lse, const int32_t *table,
                                     int32_t max_pages, const int32_t *lens, int32_t n_seqs,
                                     int32_t n_new, int32_t n_heads, int32_t window,
                                     int32_t sinks, float scale, void *workspace,
                                     size_t workspace_bytes, hipStream_t stream);
size_t f3s_cache_attend_window_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                               int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                               int32_t window, int32_t sinks);

/*
 * The same as f3s_cache_attend, but that the n_new newest tokens are a tree (a draft with
 * several continuations): token t sees the prefix, its sequence's positions before the
 * n_new, itself and its ancestors, not its siblings or what follows them.
 *   parents    device int32 [n_seqs, n_new]: the parent of token t, one of 0 .. t - 1;
 *              any other number (-1, say) for a token without one.  (A sequence with
 *              fewer drafted tokens than n_new has the last tokens of its text ahead of
 *              them, each the parent of the next, as far as they reach; tokens without a
 *              place, ahead of the sequence's start, see the prefix only)
 *   n_new      at most 256 (else F3S_ERR_UNSUPPORTED)
 *   workspace  at least f3s_cache_attend_tree_workspace_bytes(...) bytes
 * Rows are worked on as in f3s_cache_attend_window, a prefix as in f3s_cache_attend.
 */
f3s_status_t f3s_cache_attend_tree(const f3s_cache_t *cache, const void *Q, f3s_dtype_t dtype,
                                   void *O, float *lse, const int32_t *table, int32_t max_pages,
                                   const int32_t *lens, int32_t n_seqs, int32_t n_new,
                                   int32_t n_heads, const int32_t *parents,
                                   const int32_t *prefix, int32_t prefix_len, float scale,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream);
size_t f3s_cache_attend_tree_workspace_bytes(const f3s_cache_t *cache, int32_t max_pages,
                                             int32_t n_seqs, int32_t n_new, int32_t n_heads,
                                             int32_t prefix_len);

#ifdef __cplusplus
}
#endif

#endif /* F3S_CACHE_H */
