/*
 * Page tables and slot maps of a cache in pages, kept on one MI355X (gfx950) from the lengths of its sequences, C boundary.
 *
 * A sequence of L tokens needs the pages that lie in its mask as a next token sees it (arrow_attention.h): column c of its row of the table, tokens c T .. c T + T - 1,
 * where c T < L and (window == 0, or (c + 1) T > L - window, or c T < sinks).  A step takes the sequences from the lengths that the table is for, `held`, to new ones, n of whose
 * tokens, the last ones, are new:
 *   - pages of columns that were needed and are not any more go back to the list of free pages, and their entries become -1;
 *   - columns that are needed now, were not before, and begin with a new token get pages from the list, -1 where it has run out;
 *   - the place of each new token is page * T + its number in the page, or -1 where its column has no page or the table no such column.
 * A sequence that ends has length 0.  One that is shortened gives back what is behind its new end.
 *
 * The list of free pages, 1 + pages values: how many there are, then they, the last one taken first.  Pages are taken and given back in the order of the
 * sequences and of their columns, the ones that are given back so that the first of them is on top: a step there and back leaves the list as it was.  A page is in one place, of the list or
 * the table; entries of the table outside 0 .. pages - 1 are pages that are not there.
 *
 * Conventions are those of arrow.h: device pointers of the current device, work enqueued on `stream` (a hipStream_t) without waiting, nothing
 * allocated, an arrow_status code and the text in arrow_last_error().  Calls may be captured into a graph.  No atomics: results are the same every time.
 */
#ifndef ARROW_PAGES_H
#define ARROW_PAGES_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct arrow_pages_t {
  int32_t batch;         /* sequences                                                                                   */
  int32_t columns;       /* of the table; columns * page is at most 2^26, batch * columns 2^31 - 1                       */
  int32_t page;          /* tokens of a page, T: a power of two                                                         */
  int32_t window, sinks; /* of the mask                                                                                 */
  int32_t tokens;        /* new tokens of each sequence; not used with offsets                                          */
  int64_t pages;         /* of the pool, 0 .. 2^30                                                                      */
  const int32_t *offsets; /* DEVICE, batch + 1 values, or NULL: sequence b has the new tokens offsets[b] .. offsets[b+1] - 1 of `rows`; they do not fall */
  int64_t rows;          /* of `slots` with offsets                                                                     */
} arrow_pages_t;

/*
 * lengths: DEVICE, int32, batch: the new lengths.  State, DEVICE, int32: held, batch; table, batch x columns; list, 1 + pages.
 * slots: DEVICE, int64: batch x tokens, or rows with offsets; every one is written (-1 for rows that no sequence has).  NULL where there are none.
 * What columns a sequence needs goes by its length cut to 0 .. columns * T; `held` keeps the length itself, and new tokens' places count from it: those beyond the table have none.
 * Steps of offsets are cut to 0 .. rows.
 * ws: DEVICE, 256-byte aligned, at least arrow_pages_workspace_bytes(a); written, holds nothing between calls.
 * Errors: EINVAL, ETOOSMALL, EHIP.
 */
size_t arrow_pages_workspace_bytes(const arrow_pages_t *a);
int arrow_pages_step(const arrow_pages_t *a, const int32_t *lengths, int32_t *held, int32_t *table, int32_t *list, int64_t *slots, void *ws, size_t ws_bytes,
                     void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ARROW_PAGES_H */
