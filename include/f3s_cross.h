/*
 * f3s_cross.h -- dense attention of the tokens of a ragged batch to another
 * set of rows (an encoder's states), forward and backward (libf3s.so).
 *
 *     O = softmax(scale Q K^T) V   within each sequence
 *
 * Sequence b has the rows q_ptr[b] .. q_ptr[b+1] - 1 of Q and k_ptr[b] ..
 * k_ptr[b+1] - 1 of K and V.  With q_len (k_len) given, only the first
 * q_len[b] (k_len[b]) of them are there, the others are padding: never read
 * as keys, O = 0 and lse = -inf as queries, zero gradients; their contents
 * may be anything, NaN included.  A sequence without keys gives O = 0, lse =
 * -inf and zero gradients.  Query head h uses key head h / (n_heads /
 * n_kv_heads).
 */
#ifndef F3S_CROSS_H
#define F3S_CROSS_H

#include "f3s.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct f3s_cross_plan_s *f3s_cross_plan_t;

/*
 * The work of a batch of these lengths, divided among the GPU's compute
 * units; one plan serves every layer, forward and backward.
 *   q_ptr, k_ptr   HOST int32[n_seqs + 1], first 0, non-decreasing
 *   q_len, k_len   HOST int32[n_seqs] or NULL, 0 <= len[b] <= ptr[b+1] - ptr[b]
 *   n_heads        query heads, a multiple of n_kv_heads >= 1, at most 65535
 *                  (else F3S_ERR_UNSUPPORTED)
 *   d              multiple of 32, 32 <= d <= 256 (else F3S_ERR_UNSUPPORTED)
 * The forward takes 16 query rows of a key head to a workgroup where no
 * sequence has more than 8 (single tokens), else 128 (environment
 * F3S_CROSS_ROWS=16 or 128, read here, forces one).
 * The plan copies what it needs.  Synchronous on the current device's null
 * stream.  NULL on error (f3s_last_error); F3S_ERR_TOO_LARGE if the batch has
 * more than 2^31 - 2^12 rows of K, or query rows per key head, or more than 2^23
 * tiles of rows (or pieces of them).
 */
f3s_cross_plan_t f3s_cross_plan(const int32_t *q_ptr, const int32_t *k_ptr,
                                const int32_t *q_len, const int32_t *k_len, int32_t n_seqs,
                                int32_t n_heads, int32_t n_kv_heads, int32_t d);

/* Release a plan and its device memory.  NULL is a no-op. */
void f3s_cross_destroy(f3s_cross_plan_t plan);

/* Device bytes of scratch a forward (backward) call needs; 0 for a null plan.
   Host-only. */
size_t f3s_cross_forward_workspace_bytes(f3s_cross_plan_t plan);
size_t f3s_cross_backward_workspace_bytes(f3s_cross_plan_t plan);

/*
 * Forward.
 *   Q, O       device, dtype (F3S_DTYPE_F16 or F3S_DTYPE_BF16), [q_ptr[n_seqs],
 *              n_heads, d] row-major, 16-byte aligned
 *   K, V       device, dtype, [k_ptr[n_seqs], n_kv_heads, d]
 *   lse        device fp32 [q_ptr[n_seqs], n_heads] (natural logarithm)
 *   workspace  device, at least f3s_cross_forward_workspace_bytes(plan) bytes,
 *              256-byte aligned; needs no initialisation; NULL if that is 0
 *   scale      finite
 *   stream     of the plan's device (else F3S_ERR_INVALID_VALUE)
 * Inputs must be finite where they are not padding.  Outputs and workspace must
 * not overlap each other or an input.  Scores, softmax and sums in fp32 (scaled
 * scores and |V| times the number of keys have to stay below 2^127); the
 * probabilities enter the value product in dtype (fp16: relative to the row's
 * largest, one below 2^-23 keeps multiples of 2^-33), O is rounded once.
 * Asynchronous on `stream`; no allocation, no synchronisation; deterministic.
 * Calls on one plan may overlap in time, each with a workspace of its own.
 */
f3s_status_t f3s_cross_forward(f3s_cross_plan_t plan, const void *Q, const void *K,
                               const void *V, f3s_dtype_t dtype, void *O, float *lse,
                               float scale, void *workspace, size_t workspace_bytes,
                               hipStream_t stream);

/*
 * Gradients given dO = dL/dO, with O and lse from the forward:
 *   delta_i = dO_i . O_i,  dS_ij = P_ij (dO_i . V_j - delta_i),
 *   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,
 * dK and dV summed over the query heads of a key head.  dO, dQ as Q; dK, dV
 * as K; every element is written.  P comes from the scores and lse in fp32: at
 * scaled scores of 2^20 it is off by some percent, and of fp16 inputs dV may be
 * infinite from 2^24 on.  P and dS enter the products in dtype.  In fp16 P is taken
 * times 2^12, so that probabilities down to 2^-26 keep 11 bits; dS is not, and fp16
 * gradients need the usual scaling of the loss: a dS below 2^-14 loses bits.  Sums
 * in fp32, gradients rounded once.  delta comes from the rounded O: where one key
 * has nearly all of a row's probability, dS is what is left of two equal numbers
 * and keeps that rounding (2^-9 of |dO . O| in bf16).  Otherwise as the forward.
 */
f3s_status_t f3s_cross_backward(f3s_cross_plan_t plan, const void *Q, const void *K,
                                const void *V, f3s_dtype_t dtype, const void *O,
                                const void *dO, const float *lse, void *dQ, void *dK,
                                void *dV, float scale, void *workspace,
                                size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* F3S_CROSS_H */
