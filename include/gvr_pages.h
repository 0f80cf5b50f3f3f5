/*
 * gvr_pages.h -- the pages of a paged cache, handed out on the GPU (MI355X,
 * gfx950): from the tokens that each request keeps and brings, one call makes
 * the block tables, slots, positions and row starts that the rotation, the
 * cache's append, the indexer and the attention take.
 *
 * A pool is
 *   block_table [R][width] int32   page numbers of request r's tokens, page
 *                                  after page; -1 where it has none
 *   ctx_len [R] int32              tokens that request r holds
 *   free_pages [pages] int32       a stack: the free_count[0] first entries are
 *   free_count [1] int32           the numbers of the pages that nobody has
 * One step cuts request r back to keep_r tokens (rejected draft tokens; 0: the
 * request has ended) and adds n_r to it. With P the page size, ctx_r the length
 * before, keep_r = clamp(keep[r], 0, ctx_r) (ctx_r without `keep`), n_r =
 * max(new_len[r], 0), start_r = sum_{i < r} n_i and T the rows of the step's
 * buffers:
 *     more_r  = max(0, ceil((keep_r + n_r) / P) - ceil(ctx_r / P))
 *     fits_r  = start_r + n_r <= T  and  ceil((keep_r + n_r) / P) <= width
 *     served_r = fits_r and (more_r == 0 or
 *                sum of more_i over i <= r with fits_i <= free_count)
 *     ctx_r  <- keep_r + n_r if served_r, else keep_r
 * A request that is not served is cut back all the same, and gets no tokens; its
 * rows are there and marked. Pages are taken from the top of the stack, in the
 * order of requests and of their tokens; pages given back go onto it so that the
 * first of them (in the same order) is on top, and are handed out from the next
 * step on. So taking a step back (keep the old lengths, bring nothing) restores
 * the pool, the stack's order included.
 *
 * Results, each NULL if not wanted; row t = start_r + i, i < n_r, of a served
 * request is its token at position p = keep_r + i:
 *   q_start [R + 1] int32   min(start_r, T), and the sum of all
 *   taken [R] int32         n_r, 0 for a request that was not served
 *   positions [T] int32     p
 *   slots [T] int64         block_table[r][p / P] * P + p % P
 *   dense [T] int64         r * ld + p (the row of a cache [R][ld][...]), -1 where
 *                           p >= ld: the request has no such row there
 *   row_len [T] int32       p + 1: the tokens that the row sees
 * All other rows up to T (padding, requests that were not served): position 0,
 * slot -1, dense -1, row_len 0, which the append skips and the Top-K and the
 * indexer take as empty.
 *
 * Arrays are DEVICE pointers on the current HIP device, owned by the caller; the
 * structs are HOST pointers read during the call. The results depend on the
 * inputs alone (no atomics). Lengths are read with 64-bit sums; a ctx_len outside
 * [0, width * P] counts as the nearer end, a free_count outside [0, pages] too.
 * A page number outside [0, 2^31 / P) in a request's table gives slot -1.
 * Work is enqueued on `stream` as one kernel (small steps) or three; nothing is
 * allocated and nothing synchronises, so the call may be captured into a graph.
 */
#ifndef GVR_PAGES_H
#define GVR_PAGES_H

#include <stddef.h>
#include <stdint.h>

#include "gvr_topk.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gvr_page_pool {
    int32_t* block_table;   /* [requests][width] */
    int32_t* ctx_len;       /* [requests] */
    int32_t* free_pages;    /* [pages] */
    int32_t* free_count;    /* [1] */
    int64_t width;          /* pages of a request at most; width * page_size <= 2^31 - 16 */
    int64_t pages;          /* entries of free_pages, at most 2^31 - 16 */
    int32_t requests;       /* 0 .. 2^20 */
    int32_t page_size;      /* a power of two, 1 .. 65536 */
} gvr_page_pool;

typedef struct gvr_page_step_args {
    const int32_t* new_len;   /* [requests] */
    const int32_t* keep;      /* [requests] or NULL: every request keeps all it has */
    int64_t T;                /* rows of the step's buffers, 0 .. 2^31 - 16 */
    int64_t ld;               /* rows of a request in `dense` */
    int32_t* q_start;
    int32_t* taken;
    int32_t* positions;
    int64_t* slots;
    int64_t* dense;
    int32_t* row_len;
} gvr_page_step_args;

/* Bytes of workspace that a step of so many requests needs (-1 outside
 * 0 .. 2^20). */
int64_t gvr_page_step_workspace(int32_t requests);

/* One step. workspace: 16-byte aligned device memory of at least
 * gvr_page_step_workspace(requests) bytes, used by this call only while it runs
 * (no clearing needed).
 * Errors: GVR_ERR_INVALID_ARG (a NULL or misaligned required pointer, a negative
 * or bad size, with `dense` an ld below 0), GVR_ERR_TOO_LONG (sizes above their
 * limits), GVR_ERR_WORKSPACE (too little of it), GVR_ERR_HIP. With
 * requests == 0 every row is padding. */
gvr_status gvr_page_step(const gvr_page_pool* pool, const gvr_page_step_args* args, void* workspace, size_t ws_bytes,
                         void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GVR_PAGES_H */
