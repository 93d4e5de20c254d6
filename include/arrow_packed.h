/*
 * A cache of keys and values in 4 bits, and the attention of arrow_attention.h for single tokens over it, on one MI355X (gfx950), C boundary.
 *
 * A row of `dim` elements becomes codes of 4 bits and a scale for every 32 of them (the microscaled form e2m1 with scales e8m0): a code is a sign (its highest bit)
 * and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 in that order, a scale the byte e for 2^(e - 127), an element their product.  Written, the scale is the
 * smallest power of two of which no element's size is more than seven times, within 2^-126 .. 2^125 (float16: up to 2^13), the code the nearest one, of two the one whose
 * lowest bit is 0, and 6 for all above: no element is further off than half of the largest step, unless that scale was cut (of the type's largest elements one may be off by nearly
 * all of it: 65504 in float16 becomes 49152).  Elements that are not finite make their 32 ones NaN (e = 255).
 *
 * The block of a page of T tokens and one head, (dim + dim/16) T bytes:
 *     keys' codes     T x dim/2                       byte i of a row holds elements 2 i (low half) and 2 i + 1
 *     values' codes   T/4 x 16 x 4 x dim/32           those of four tokens together, in sixteen pieces of a row each
 *     keys' scales    T x dim/32
 *     values' scales  T/4 x dim/32 x 4
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without waiting, nothing
 * allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.  Scores, softmax statistics and all sums are held in 32
 * bits; a probability goes into the product as two numbers of the operands' type, off by 2^-16 (float16: 2^-22) of itself, elements of the cache are exact in that type.  No atomics: results are bitwise reproducible.
 */
#ifndef ARROW_PACKED_H
#define ARROW_PACKED_H

#include <stddef.h>
#include <stdint.h>

#include "arrow_attention.h" /* arrow_dtype, arrow_strides_t */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct arrow_packed_t {
  int32_t dtype;             /* ARROW_BF16 or ARROW_F16: of q, k, v, o; a cache is read in the type that it was written in */
  int32_t batch;             /* sequences (decode)                                                                         */
  int32_t q_heads, kv_heads; /* q_heads (decode) a multiple of kv_heads                                                    */
  int32_t dim;               /* of a head: 32, 64 or 128                                                                   */
  int32_t window, sinks;     /* the mask of arrow_attention.h (decode)                                                     */
  float scale;               /* of the scores (decode)                                                                     */
  int32_t page;              /* tokens of a page: a power of two, 16 or more                                               */
  int32_t columns;           /* of `table` (decode)                                                                        */
  int64_t pages;             /* of the pool                                                                                */
  int64_t max_len;           /* longest sequence; only how the work is split goes by it (decode)                           */
  int64_t page_step, head_step; /* bytes between blocks of the pool, multiples of 16                                       */
  const int32_t *table;      /* as arrow_cache_t has it (decode)                                                              */
  const int32_t *lengths;
} arrow_packed_t;

/*
 * Write `tokens` rows, k and v: tokens x kv_heads x dim by their strides (sequence unused), to the places slots[i] = page * T + token (DEVICE, int64), and read them from there.
 * Slots outside the pool are places that are not there: nothing is written for them, and zeros are read.  Two rows written to one place leave parts of both.  What is written, here
 * and below, overlaps neither itself nor another operand.
 * Errors: EINVAL, EHIP.
 */
int arrow_packed_append(const arrow_packed_t *c, int64_t tokens, const void *k, const void *v, arrow_strides_t ks, arrow_strides_t vs, const int64_t *slots,
                        void *pool, void *stream);
int arrow_packed_read(const arrow_packed_t *c, int64_t tokens, const int64_t *slots, const void *pool, void *k, void *v, arrow_strides_t ks, arrow_strides_t vs,
                      void *stream);

/*
 * o of one query per sequence, at position lengths[b] - 1, as arrow_attention_decode has it.  k, v: the new token's key and value (token step unused), which are
 * written to their place first, or both NULL where they are in the pool.  batch * q_heads is at most 2^24 - 1.  A page that is not there, or an idle sequence, is as there.
 * ws: DEVICE, 256-byte aligned, at least arrow_packed_decode_workspace_bytes(c) (which may be 0); written, holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_packed_decode_workspace_bytes(const arrow_packed_t *c);
int arrow_packed_decode(const arrow_packed_t *c, const void *q, arrow_strides_t qs, const void *k, const void *v, arrow_strides_t ks, arrow_strides_t vs,
                        void *pool, void *o, arrow_strides_t os, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_PACKED_H */
