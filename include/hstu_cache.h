/*
 * hstu_cache.h -- C ABI of the paged key-value cache of the jagged HSTU attention
 * and of the attention of one new token over it (serving).
 *
 * A sequence recommender that serves long histories keeps every sequence's keys,
 * values and timestamps from step to step.  Here they lie in pages of page_size
 * tokens; a sequence is a slot with a table of pages and a length.  Sequences may
 * share pages (beams of one prompt): refs counts, for every page, the table entries
 * that name it, and a page is free exactly when its count is 0.
 *
 * The bookkeeping lives in device memory and is done by the calls below, so that no
 * step waits for the host.  Every result is determined by the arguments: a call
 * takes the lowest free pages, row by row.
 *
 * Pointers and streams.  Every pointer inside hstu_cache and every array argument
 * is a DEVICE pointer on the current HIP device; the caller owns all memory.  Calls
 * never allocate and never synchronise: each enqueues its kernels on `stream` (a
 * hipStream_t; NULL = the default stream) and returns, and may be captured into a
 * graph.  Calls on one cache must be ordered by the caller (one stream, or events),
 * except that hstu_paged_attn_fwd calls may overlap each other, with a workspace
 * each.
 *
 * Entries that name no slot or page.  Slot indices are checked on the device
 * against [0, slots), pages against [0, num_pages), and lengths against the table;
 * what is outside is left out (a row is skipped, a token adds nothing) and never
 * read or written.
 *
 * Return codes as in hstu_jagged.h; hstu_last_error() describes a failure.
 */
#ifndef HSTU_CACHE_H
#define HSTU_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "hstu_jagged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bits of hstu_cache.status; calls only ever set them (hstu_cache_clear clears). */
#define HSTU_CACHE_FULL 0x1       /* extend: a row found too few pages, or columns  */
#define HSTU_CACHE_BAD_SLOT 0x2   /* a slot index outside [0, slots)                */
#define HSTU_CACHE_TWICE 0x4      /* extend, fork: a slot named twice as target     */
#define HSTU_CACHE_BAD_COUNT 0x8  /* extend: a negative count                       */

typedef struct {
    hstu_dtype dtype;            /* of k, v (HSTU_BF16: d 64 or 128)         */
    int32_t layers;              /* >= 1                                     */
    int32_t num_pages;           /* >= 1; num_pages * page_size < 2^31       */
    int32_t page_size;           /* tokens: a power of two, at most 1024     */
    int32_t H, d;                /* as in hstu_jagged.h                      */
    int32_t slots;               /* >= 1                                     */
    int32_t max_pages;           /* columns of a table; max_pages *
                                    page_size < 2^31                         */
    void *k, *v;                 /* [layers][num_pages][page_size][H][d]     */
    int64_t *ts;                 /* [num_pages][page_size], or NULL          */
    int32_t *tables;             /* [slots][max_pages]; -1: no page          */
    int32_t *lens;               /* [slots] tokens                           */
    int32_t *refs;               /* [num_pages] table entries naming it      */
    int32_t *status;             /* [1] HSTU_CACHE_* bits                    */
} hstu_cache;

/* Bytes of device workspace (256-byte aligned) of the calls that take one; 0 for
 * invalid sizes. */
size_t hstu_cache_workspace_bytes(const hstu_cache *c);

/* Empties the cache: no pages in any table, lengths, counts and status 0 (k, v and
 * ts are left as they are).  A new cache is cleared before its first use. */
int hstu_cache_clear(const hstu_cache *c, void *stream);

/* Room for counts[r] more tokens at the end of sequence slot_ids[r], r < n <= slots:
 * tables and lengths grow, start[r] receives the position of the first new token.
 * A last page with room that other tables name too is copied first (its tokens, all
 * layers), so that what the sequence writes is its own; whether it is shared is
 * decided on the counts before the call.  A row is refused, with start[r] = -1 and
 * nothing else changed for it, when its slot is no slot or is named by an earlier
 * row, its count is negative, its table has too few columns, or when it needs pages
 * and the rows up to it (those refused for want of pages included) need more than
 * there are. */
int hstu_cache_extend(const hstu_cache *c, const int32_t *slot_ids,
                      const int32_t *counts, int32_t n, int32_t *start,
                      void *workspace, size_t workspace_bytes, void *stream);

/* Writes one layer's rows: rows row_offsets[r] .. row_offsets[r+1]-1 of k and v
 * ([total_rows][H][d]) become the tokens from start[r] on of sequence slot_ids[r]
 * (start as extend returned it; rows with start[r] < 0 are skipped).  row_offsets
 * (int64, n + 1) as seq_offsets in hstu_jagged.h; of a row that holds more than
 * max_new tokens the first max_new are written.  With timestamps ([total_rows], and c->ts) those are written too: once a
 * step, with any of its layers.  No two rows name the same tokens. */
int hstu_cache_write(const hstu_cache *c, int32_t layer, const void *k,
                     const void *v, const int64_t *timestamps,
                     const int32_t *slot_ids, const int32_t *start,
                     const int64_t *row_offsets, int32_t n, int64_t total_rows,
                     int32_t max_new, void *stream);

/* dst[r] becomes a sequence with the tokens that src[r] has before the call, on
 * shared pages, for all rows at once (so src may permute dst: the reordering of
 * beams); what dst[r] held is freed.  Rows with a slot that is none, or whose dst
 * an earlier row names, are skipped. */
int hstu_cache_fork(const hstu_cache *c, const int32_t *src, const int32_t *dst,
                    int32_t n, void *workspace, size_t workspace_bytes,
                    void *stream);

/* Ends the sequences slot_ids[r] (naming one twice frees it once). */
int hstu_cache_free(const hstu_cache *c, const int32_t *slot_ids, int32_t n,
                    void *stream);

/* Moves the pages in use to the front of their pools: with L pages in use, the
 * k-th of those at or behind page L moves to the k-th free page before it; tables
 * and counts follow.  *live (device int32) receives L. */
int hstu_cache_compact(const hstu_cache *c, int32_t *live, void *workspace,
                       size_t workspace_bytes, void *stream);

/* Attention of one new token of every sequence over the cache.  Row r is the last
 * token of sequence slot_ids[r], whose own key, value (and timestamp) are in the
 * cache already, at position i = lens - 1:
 *
 *   o_r = sum over seen j <= i of silu(s_ij) / N v_j,  y_r = LayerNorm(o_r) * u_r
 *
 * with s_ij, N = max_len, biases, LayerNorm and precision as in hstu_jagged.h, and
 * every j <= i seen (win = NULL) or those of a window and the first tokens
 * (hstu_window): what hstu_jagged_attn_fwd gives for the last token of the same
 * history, up to the order of sums.  rab->timestamps is not used: with time_w the
 * cache's ts must be there.  q [rows][H][d], u, y [rows][H*d], o [rows][H][d].
 * lens <= max_len is the caller's contract (entries of a bias table that lie
 * outside it read as 0).  A sequence without tokens, or a row that names no slot,
 * has o = 0, y = 0.  A slot may be named by several rows.
 *
 * A sequence's tokens are cut into chunks, as long for all sequences and such that
 * the device is filled, a work-group each (and for each group of heads); their sums
 * (float32) are added in order by a second launch, which also normalises.  Bits
 * depend on the batch (its lengths set the chunks), not on timing. */
typedef struct {
    void *y;                     /* [rows][H*d]                              */
    void *o;                     /* [rows][H][d]                             */
    void *workspace;             /* device scratch, 256-byte aligned         */
    size_t workspace_bytes;      /* >= hstu_paged_attn_workspace_bytes(..)   */
} hstu_paged_out;

size_t hstu_paged_attn_workspace_bytes(const hstu_cache *c, int32_t rows);

int hstu_paged_attn_fwd(const void *q, const void *u, const hstu_cache *c,
                        int32_t layer, const int32_t *slot_ids, int32_t rows,
                        int32_t max_len, const hstu_rab *rab,
                        const hstu_window *win, hstu_paged_out *out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HSTU_CACHE_H */
