/*
 * f3s_pages.h -- the page tables of a paged cache (f3s_cache.h), kept on the device:
 * pages given to sequences that grow, taken back from those that shrink, and the places
 * of the newest tokens (libf3s.so).
 *
 * The pool is a list of free pages on the device: `free_pages` has room for all n_pages
 * of them, the first *n_free are free.  A sequence of `len` tokens holds the pages that
 * the first ceil(len / page_size) entries of its row of the table name; the others may
 * hold anything.  No page is in the pool and in the table, or twice in one of them
 * (pages that sequences share, such as those of a common prefix, are not the pool's).
 */
#ifndef F3S_PAGES_H
#define F3S_PAGES_H

#include "f3s.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bring the table from lengths `lens` to lengths `new_lens`.
 *
 * First every sequence that shrinks gives the pages that it no longer needs back: they
 * are appended to the pool in the order of sequences and entries, and their entries
 * become -1 (an entry outside [0, n_pages) is no page and is not appended).  Then every
 * sequence that grows takes the pages that it needs: of `need` pages in all, the last
 * min(need, *n_free) of the pool are handed out, in the pool's order, in the order of
 * sequences and entries.  Where they do not suffice, the last sequences' entries become
 * -1 and their lengths got_lens[b] end with the last page that they got; a caller that
 * goes on with got_lens keeps the table whole.  Growing by a call and shrinking back by
 * the next one restores the pool, order included.
 *
 *   free_pages, n_free   device int32 [n_pages], [1]; updated.  A count outside 0 ..
 *                        n_pages counts as the nearest of them
 *   table                device int32 [n_seqs, max_pages]; updated
 *   lens, new_lens       device int32 [n_seqs]; below 0 as 0, and beyond the table as its
 *                        room, max_pages * page_size (at most 2^30, else
 *                        F3S_ERR_TOO_LARGE)
 *   got_lens             device int32 [n_seqs], the lengths that the table then holds:
 *                        new_lens where pages sufficed
 *   slots                device int64 [n_seqs, n_new], the places of the n_new newest
 *                        tokens: of position p = new_lens[b] - n_new + t, page *
 *                        page_size + p % page_size; -1 where p is below 0 or at least
 *                        got_lens[b], or its entry is no page.  NULL if n_new is 0
 *   page_size            16, 32, 64, 128 or 256 (else F3S_ERR_UNSUPPORTED)
 *   workspace            device, at least f3s_pages_assign_workspace_bytes(n_seqs,
 *                        max_pages, n_new) bytes, 16-byte aligned; needs no
 *                        initialisation; NULL if that is 0
 * What is written must not overlap anything else of the call.  F3S_ERR_TOO_LARGE beyond
 * 2^24 sequences or 2^30 new tokens.  Whole numbers in a fixed order: deterministic.
 * Asynchronous on `stream`; no allocation, no synchronisation: it can be captured, and a
 * replay takes its lengths from the device.  Calls on one pool or table follow one
 * another.
 */
f3s_status_t f3s_pages_assign(int32_t *free_pages, int32_t *n_free, int32_t n_pages,
                              int32_t *table, int32_t max_pages, const int32_t *lens,
                              const int32_t *new_lens, int32_t *got_lens, int64_t *slots,
                              int32_t n_seqs, int32_t n_new, int32_t page_size,
                              void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Device bytes of scratch such a call needs (0 also for sizes that it refuses).
   Host-only. */
size_t f3s_pages_assign_workspace_bytes(int32_t n_seqs, int32_t max_pages, int32_t n_new);

#ifdef __cplusplus
}
#endif

#endif /* F3S_PAGES_H */
