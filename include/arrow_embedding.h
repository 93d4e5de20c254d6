/*
 * Embedding lookup with scaling, and its gradient, on one MI355X (gfx950), C boundary.
 *
 *     Y_t = scale W[ids_t]            dW_v = scale sum_{t: ids_t = v} dY_t
 *
 * the product of a one-hot matrix and of its transpose with a dense one.  An id outside 0 .. rows-1 (padding) gives Y_t = 0 and adds to no row.
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without
 * waiting, nothing allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.
 * The gradient sorts the tokens by id and adds up each row's in their order, in 32 bits: no atomics on sums, results are bitwise reproducible.
 */
#ifndef ARROW_EMBEDDING_H
#define ARROW_EMBEDDING_H

#include <stddef.h>
#include <stdint.h>

#include "arrow_attention.h" /* arrow_dtype */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct arrow_embedding_t {
  int32_t dtype;       /* of W, Y and dY: ARROW_F32, ARROW_BF16 or ARROW_F16      */
  int32_t grad_dtype;  /* of dW: `dtype` or ARROW_F32                              */
  int32_t id_bytes;    /* 4 or 8: ids are int32 or int64                           */
  int32_t columns;     /* >= 1                                                     */
  int64_t rows;        /* of W, 1 .. 2^31 - 2                                      */
  int64_t tokens;      /* 0 .. 2^31 - 1 (gradient: 2^30)                           */
  int64_t w_stride, y_stride; /* elements between rows of W (and dW), of Y (and dY), >= columns */
  float scale;
} arrow_embedding_t;

/* Y = scale E W.  Y must not overlap W.  Errors: EINVAL, EHIP. */
int arrow_embedding_forward(const arrow_embedding_t *e, const void *W, const void *ids, void *Y, void *stream);

/*
 * dW = scale E^T dY: every row of dW is written (rows without tokens become 0); it must not overlap dY.
 * ws: DEVICE, 256-byte aligned, at least arrow_embedding_workspace_bytes(e); written (not by calls of few tokens), holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_embedding_workspace_bytes(const arrow_embedding_t *e);
int arrow_embedding_backward(const arrow_embedding_t *e, const void *dY, const void *ids, void *dW, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_EMBEDDING_H */
