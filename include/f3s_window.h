/*
 * f3s_window.h -- causal self-attention of a ragged batch in which a token sees the
 * newest `window` tokens and the first `sinks` ones, forward and backward (libf3s.so).
 *
 *     O = softmax(scale Q K^T) V   over the keys that a token sees
 *
 * Sequence b has the rows k_ptr[b] .. k_ptr[b+1] - 1 of K and V, at the positions 0, 1,
 * ..., and the rows q_ptr[b] .. q_ptr[b+1] - 1 of Q, which are its newest: of nq query
 * and nk key rows, query row i stands at position nk - nq + i.  The token at position p
 * sees position j <= p if p - j < window (itself, then, and the window - 1 before it)
 * or j < sinks.  A window as long as the sequence is plain causal attention.  A token
 * that sees nothing (a position below 0, where there are more query rows than keys; a
 * window of 0 without sinks) gives O = 0, lse = -inf and zero gradients.
 *
 * With q_len (k_len) given, only the first q_len[b] (k_len[b]) rows of a sequence are
 * there, the others are padding: never read as keys, O = 0 and lse = -inf as queries,
 * zero gradients; their contents may be anything, NaN included.  Query head h uses key
 * head h / (n_heads / n_kv_heads).
 */
#ifndef F3S_WINDOW_H
#define F3S_WINDOW_H

#include "f3s.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct f3s_window_plan_s *f3s_window_plan_t;

/*
 * The work of a batch of these lengths, divided among the GPU's compute units; one plan
 * serves every layer, forward and backward.
 *   q_ptr, k_ptr   HOST int32[n_seqs + 1], first 0, non-decreasing
 *   q_len, k_len   HOST int32[n_seqs] or NULL, 0 <= len[b] <= ptr[b+1] - ptr[b]
 *   n_heads        query heads, a multiple of n_kv_heads >= 1, at most 65535
 *                  (else F3S_ERR_UNSUPPORTED)
 *   d              multiple of 32, 32 <= d <= 256 (else F3S_ERR_UNSUPPORTED)
 *   window, sinks  >= 0; from 2^30 on as 2^30
 * The plan copies what it needs.  Synchronous on the current device's null stream.
 * NULL on error (f3s_last_error); F3S_ERR_TOO_LARGE if the batch has more than 2^31 -
 * 2^12 rows of K, or query rows per key head, or more than 2^23 tiles of 128 rows (or
 * pieces of them).
 */
f3s_window_plan_t f3s_window_plan(const int32_t *q_ptr, const int32_t *k_ptr,
                                  const int32_t *q_len, const int32_t *k_len, int32_t n_seqs,
                                  int32_t n_heads, int32_t n_kv_heads, int32_t d,
                                  int32_t window, int32_t sinks);

/* Release a plan and its device memory.  NULL is a no-op. */
void f3s_window_destroy(f3s_window_plan_t plan);

/* Device bytes of scratch a forward (backward) call needs; 0 for a null plan.
   Host-only. */
size_t f3s_window_forward_workspace_bytes(f3s_window_plan_t plan);
size_t f3s_window_backward_workspace_bytes(f3s_window_plan_t plan);

/*
 * Forward.  Arguments, precision and conditions as f3s_cross_forward (f3s_cross.h):
 * Q, O [q_ptr[n_seqs], n_heads, d], K, V [k_ptr[n_seqs], n_kv_heads, d] in F16 or BF16,
 * lse fp32 [q_ptr[n_seqs], n_heads].  Inputs must be finite where they are not padding:
 * a row of K or V that is not may reach tokens before it too.
 */
f3s_status_t f3s_window_forward(f3s_window_plan_t plan, const void *Q, const void *K,
                                const void *V, f3s_dtype_t dtype, void *O, float *lse,
                                float scale, void *workspace, size_t workspace_bytes,
                                hipStream_t stream);

/*
 * Gradients given dO = dL/dO, with O and lse from the forward, as f3s_cross_backward:
 * dK and dV summed over the query heads of a key head and over the tokens that see the
 * key; every element is written.  Deterministic, without atomics.
 */
f3s_status_t f3s_window_backward(f3s_window_plan_t plan, const void *Q, const void *K,
                                 const void *V, f3s_dtype_t dtype, const void *O,
                                 const void *dO, const float *lse, void *dQ, void *dK,
                                 void *dV, float scale, void *workspace,
                                 size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* F3S_WINDOW_H */
