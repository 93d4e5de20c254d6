/*
 * Attention under an arrow-shaped mask on one MI355X (gfx950), C boundary.
 *
 * Of a sequence with Lq queries and Lk keys, query i stands at position p = i + Lk - Lq, and key j is visible to it where
 *
 *     j <= p  and  (window == 0  or  j > p - window  or  j < sinks):
 *
 * a band of `window` keys and a first block column of `sinks` keys.  It is the sampled product of arrow.h over that
 * pattern, a softmax over each row's entries, and the product with the values, in one pass:
 *
 *     s(i,j) = scale <q_i, k_j>,   lse_i = log sum_j exp s(i,j),   o_i = sum_j exp(s(i,j) - lse_i) v_j
 *
 * over the visible j.  A row without any gives o = 0 and lse = -infinity, and no gradient.  What keys and values hold
 * where a query does not see them, NaN and infinities among it, does not touch its results or its gradient, nor do queries and gradients of
 * results touch those of keys that they do not see; what lies behind a sequence's end is not read.  A call in which results are not finite goes through their
 * tiles a second time.
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without
 * waiting, nothing allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.
 * No atomics: results are bitwise reproducible.  Scores, softmax statistics and all sums are held in 32 bits; what goes into a matrix
 * instruction (probabilities, gradients of scores) is rounded to the operands' type first; gradients in float16 by the size of d_o, so that small ones
 * keep its precision.
 */
#ifndef ARROW_ATTENTION_H
#define ARROW_ATTENTION_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum arrow_dtype {
  ARROW_F32 = 0, /* embedding only */
  ARROW_BF16 = 1,
  ARROW_F16 = 2
} arrow_dtype;

/* Steps between neighbours of an operand, in elements; the elements of a head lie next to each other. */
typedef struct arrow_strides_t {
  int64_t sequence; /* not used with offsets: the tokens of all sequences follow each other */
  int64_t token;
  int64_t head;
} arrow_strides_t;

typedef struct arrow_attention_t {
  int32_t dtype;             /* ARROW_BF16 or ARROW_F16: of q, k, v, o and their gradients                        */
  int32_t batch;             /* sequences, >= 0                                                                    */
  int32_t q_heads, kv_heads; /* q_heads a multiple of kv_heads; query head h reads key head h / (q_heads/kv_heads) */
  int32_t dim;               /* of a head: 8, 16, ..., 128                                                         */
  int32_t q_len, k_len;      /* tokens of every sequence; with offsets: at least those of the longest one          */
  int32_t window, sinks;     /* >= 0; window 0 = no window                                                         */
  float scale;               /* of the scores, positive and finite                                                 */
  /* Ragged batches: DEVICE, batch + 1 values each, or both NULL.  Sequence b has the tokens q_offsets[b] .. q_offsets[b+1]-1
   * of the q_tokens ones there are, and likewise keys.  Values outside 0 .. tokens and steps of less than 0 or more than q_len (k_len)
   * are cut to that; sequences must not overlap. */
  const int32_t *q_offsets, *k_offsets;
  int64_t q_tokens, k_tokens;
  arrow_strides_t q, k, v, o;     /* all multiples of 8, as the addresses are of 16 bytes; token steps within 0 .. 2^24 */
  arrow_strides_t d_o, dq, dk, dv; /* gradients; arrow_attention_backward only                                           */
} arrow_attention_t;

/*
 * o, lse of the formulas above.  lse: fp32, batch x q_heads x q_len (with offsets: q_heads x q_tokens), contiguous, or NULL.
 * Outputs must not overlap inputs.  Tokens that no sequence has keep what they hold.
 * Errors: EINVAL, EHIP.
 */
int arrow_attention_forward(const arrow_attention_t *a, const void *q, const void *k, const void *v, void *o, float *lse, void *stream);

/*
 * The same with a workspace, in which few queries of many keys have the keys cut over several workgroups.
 * ws: DEVICE, 256-byte aligned, at least arrow_attention_forward_split_bytes(a), which is 0 where nothing is cut; written, holds nothing
 * between calls.  Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_attention_forward_split_bytes(const arrow_attention_t *a);
int arrow_attention_forward_split(const arrow_attention_t *a, const void *q, const void *k, const void *v, void *o, float *lse, void *ws,
                                  size_t ws_bytes, void *stream);

/*
 * Gradients of the forward call with the same arguments, for the gradient d_o of its o (lse takes none):
 *     P(i,j) = exp(s(i,j) - lse_i),  dS(i,j) = P(i,j) (<do_i, v_j> - <do_i, o_i>),
 *     dq_i = scale sum_j dS(i,j) k_j,  dk_j = scale sum_i dS(i,j) q_i,  dv_j = sum_i P(i,j) do_i,
 * keys and values of a head that several query heads share summed over them.  o and lse are the forward call's.
 * ws: DEVICE, 256-byte aligned, at least arrow_attention_workspace_bytes(a); written, holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_attention_workspace_bytes(const arrow_attention_t *a);
int arrow_attention_backward(const arrow_attention_t *a, const void *q, const void *k, const void *v, const void *o, const float *lse,
                             const void *d_o, void *dq, void *dk, void *dv, void *ws, size_t ws_bytes, void *stream);

/* A cache of keys and values in pages, shared by all sequences of a batch. */
typedef struct arrow_cache_t {
  int32_t dtype;
  int32_t batch;
  int32_t q_heads, kv_heads, dim;
  int32_t window, sinks;
  float scale;
  int32_t page;              /* tokens of a page, a power of two                                                     */
  int32_t columns;           /* of `table`                                                                           */
  int64_t pages;             /* of each pool                                                                         */
  int64_t max_len;           /* longest sequence; only how the work is split goes by it                              */
  int64_t k_page, k_token, k_head; /* steps within the pool of keys, in elements, multiples of 8                     */
  int64_t v_page, v_token, v_head;
  const int32_t *table;      /* DEVICE, batch x columns: token t of sequence b lies in page table[b][t / page], at t % page.
                                Entries outside 0 .. pages-1 are pages that are not there: their keys are invisible, and
                                nothing is written to them.  Entries that no query sees are not read.                   */
  const int32_t *lengths;    /* DEVICE, batch: tokens of each sequence, the new ones among them; 0 = an idle one, o = 0.
                                More than the table has room for are cut to that.                                       */
} arrow_cache_t;

/*
 * Write `tokens` new keys and values per sequence to its last places, lengths[b] - tokens .. lengths[b] - 1 (places before
 * the first one, and those that the table has no room for, are left out).  k, v: batch x tokens x kv_heads x dim by their strides.  Errors: EINVAL, EHIP.
 */
int arrow_cache_append(const arrow_cache_t *c, int32_t tokens, const void *k, const void *v, arrow_strides_t ks, arrow_strides_t vs,
                       void *k_pool, void *v_pool, void *stream);

/*
 * o of one query per sequence, at position lengths[b] - 1.  q, o: batch x q_heads x dim by their strides (token unused).
 * k, v: the new token's key and value (token unused), which the call writes to its place first, or both NULL where they are in the pools.
 * Of a sequence longer than the table has room for, they are left out: nothing is written, and o is that of the keys that are there.
 * ws: DEVICE, 256-byte aligned, at least arrow_attention_decode_workspace_bytes(c) (which may be 0); written, holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_attention_decode_workspace_bytes(const arrow_cache_t *c);
int arrow_attention_decode(const arrow_cache_t *c, const void *q, arrow_strides_t qs, const void *k, const void *v, arrow_strides_t ks,
                           arrow_strides_t vs, void *k_pool, void *v_pool, void *o, arrow_strides_t os, void *ws, size_t ws_bytes,
                           void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_ATTENTION_H */
