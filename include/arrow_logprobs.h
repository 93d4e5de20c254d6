/*
 * Log probabilities of given tokens, entropies and the most likely tokens of rows of logits, and the gradient, on one MI355X (gfx950), C boundary.
 *
 * Of a row x of `vocabulary` logits and its target t, over all j:
 *
 *     lse = log sum_j exp(scale x_j),   p_j = exp(scale x_j - lse),   logp = scale x_t - lse,   H = lse - sum_j p_j scale x_j
 *
 * and the `top` largest logits in falling order, of equal ones the lower index first: their indices j and scale x_j - lse.  A target outside
 * 0 .. vocabulary - 1 (padding) has logp = 0 and no gradient of logp.  Logits of -infinity are tokens that cannot be: p = 0.  A row of nothing else has lse =
 * logp = -infinity (of its top, too), H = 0 and no gradient; one with NaN or +infinity has NaN in lse, logp (but of padding), H, top_logp and its gradient.  NaN counts as the largest
 * logit.
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without waiting, nothing
 * allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.  All statistics are held in 32 bits.  Results are bitwise
 * reproducible.
 */
#ifndef ARROW_LOGPROBS_H
#define ARROW_LOGPROBS_H

#include <stddef.h>
#include <stdint.h>

#include "arrow_attention.h" /* arrow_dtype */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct arrow_logprobs_t {
  int32_t dtype;       /* of the logits and their gradient: ARROW_F32, ARROW_BF16 or ARROW_F16 */
  int32_t target_bytes; /* 4 or 8: targets are int32 or int64                                   */
  int32_t top;         /* 0 .. 32, at most vocabulary                                          */
  int32_t vocabulary;  /* 1 .. 2^30                                                            */
  int64_t rows;        /* 0 .. 2^31 - 1                                                        */
  int64_t stride, d_stride; /* elements between rows of the logits, of their gradient, >= vocabulary */
  float scale;         /* of the logits (1 / temperature), positive and finite                 */
} arrow_logprobs_t;

/*
 * logp, entropy, lse: fp32, rows each.  stats: fp32, rows x 2, 8-byte aligned, for the gradient: a logit near the largest, and lse less scale times that.  top_logp (fp32), top_ids (int64): rows x top, contiguous; NULL where top is 0.
 * ws: DEVICE, 256-byte aligned, at least arrow_logprobs_workspace_bytes(a), which is 0 where rows are not cut; written, holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_logprobs_workspace_bytes(const arrow_logprobs_t *a);
int arrow_logprobs_forward(const arrow_logprobs_t *a, const void *logits, const void *targets, float *logp, float *entropy, float *lse, float *stats,
                           float *top_logp, int64_t *top_ids, void *ws, size_t ws_bytes, void *stream);

/*
 * d_logits for the gradients d_logp and d_entropy (fp32, rows each; either may be NULL for none), with the forward call's stats and entropy:
 *     d x_j = scale (d_logp ([j = t] - p_j) - d_entropy p_j (log p_j + H)).
 * d_logits may be logits where the rows are as far apart.  entropy may be NULL where d_entropy is.  Errors: EINVAL, EHIP.
 */
int arrow_logprobs_backward(const arrow_logprobs_t *a, const float *d_logp, const float *d_entropy, const void *logits, const void *targets,
                            const float *stats, const float *entropy, void *d_logits, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_LOGPROBS_H */
