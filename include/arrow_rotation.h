/*
 * Norms of queries and keys for each head, with the rotation by position in the same pass, on one MI355X (gfx950), C boundary.
 *
 * Of a head x of `dim` elements at position p, with weights w (the same for all heads of queries, or of keys):
 *
 *     r = 1 / sqrt(mean_d x_d^2 + eps),   u_d = r x_d w_d,   y = R(p) u
 *
 * R turns pair i of the first `rotary` elements by the angle 2 pi p turns[i]:  (a, b) -> (a cos - b sin, b cos + a sin).  Pair i are elements i and
 * i + rotary/2, or (interleaved) 2 i and 2 i + 1; elements from `rotary` on stay as u has them.  It is what goes into the attention of
 * arrow_attention.h as q and k.
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without waiting, nothing
 * allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.  Norms, rotations and sums are held in 32
 * bits and rounded once; an angle is reduced to its part of a turn in 64 bits, at any position.  No atomics: results are bitwise reproducible.
 */
#ifndef ARROW_ROTATION_H
#define ARROW_ROTATION_H

#include <stddef.h>
#include <stdint.h>

#include "arrow_attention.h" /* arrow_dtype, arrow_strides_t */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct arrow_rotation_t {
  int32_t dtype;             /* of q, k, results and gradients: ARROW_F32, ARROW_BF16 or ARROW_F16                 */
  int32_t weight_dtype;      /* of the weights and their gradients: `dtype` or ARROW_F32                            */
  int32_t batch, tokens;     /* sequences, and tokens of each; together at most 2^31 - 1                            */
  int32_t q_heads, kv_heads; /* >= 1                                                                                */
  int32_t dim;               /* of a head: 8, 16, ..., 256                                                          */
  int32_t rotary;            /* elements that are rotated: 0, 16, 32, ... up to dim                                 */
  int32_t interleaved;       /* 0 or 1                                                                              */
  float eps;                 /* >= 0, finite                                                                        */
  int32_t position_bytes;    /* 4 or 8: positions are int32 or int64                                                */
  const void *positions;     /* DEVICE, batch x tokens, contiguous; NULL: 0, 1, ... in each sequence                */
  int64_t shift;             /* added to every position                                                             */
  const double *turns;       /* DEVICE, rotary / 2: turns per position of each pair (NULL where rotary is 0)        */
  arrow_strides_t q, k, q_out, k_out;  /* steps in elements, not negative; addresses and steps are multiples of 16 bytes */
  arrow_strides_t dq, dk;              /* gradients of q and k; those of the results have q_out's and k_out's.  Backward only */
} arrow_rotation_t;

/*
 * q_out, k_out: y of q and k.  wq, wk: DEVICE, dim weights each, or both NULL for ones.  q_out may be q where their steps are the same, and k_out k; otherwise what is
 * written overlaps nothing (views of one tensor with the same steps, such as queries and keys of one projection, lie apart where their elements do).
 * Errors: EINVAL, EHIP.
 */
int arrow_rotation_forward(const arrow_rotation_t *a, const void *q, const void *k, const void *wq, const void *wk, void *q_out, void *k_out, void *stream);

/*
 * Gradients of the forward call with the same arguments, for the gradients d_q_out and d_k_out of its results.  With n = r x and g = R(p)^T dy:
 *     dx = r (w g - n mean_d(w g n)),   dw = sum over tokens and heads of g n.
 * dq may be d_q_out where their steps are the same, and dk d_k_out.  dwq, dwk: DEVICE, dim each, or both NULL where they are not asked for.
 * ws: DEVICE, 256-byte aligned, at least arrow_rotation_workspace_bytes(a); written, holds nothing between calls (not used without dwq).
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_rotation_workspace_bytes(const arrow_rotation_t *a);
int arrow_rotation_backward(const arrow_rotation_t *a, const void *d_q_out, const void *d_k_out, const void *q, const void *k, const void *wq,
                            const void *wk, void *dq, void *dk, void *dwq, void *dwk, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_ROTATION_H */
