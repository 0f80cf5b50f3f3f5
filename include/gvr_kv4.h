/*
 * gvr_kv4.h -- a paged key / value cache held in 4 bits on MI355X (gfx950):
 * appending tokens (keys rotated on the way), reading them back, and
 * attention over the cache -- over every token of a sequence, or over the
 * tokens that a Top-K selected.
 *
 * Number format: 32 consecutive elements of a head share a power-of-two scale
 * 2^e (one E8M0 byte, e + 127) and are 4-bit E2M1 codes: sign and one of
 * 0, 1/2, 1, 3/2, 2, 3, 4, 6 times the scale; the even element is in the low
 * four bits of its byte. 4.25 bits per element. Appending takes the least
 * e >= -126 with max|x| <= 7 * 2^e, so no element is further than half a step
 * from its code (6 < |x| / 2^e <= 7 rounds to 6), and rounds x / 2^e to the
 * nearest code, ties to the even code. A block that holds an infinity or a
 * NaN gets the scale byte 255 and reads back as NaN.
 *
 * Cache layout: data [pages][page_size][record]: a token's record is
 *     key codes    [kv_heads][head_dim / 2]
 *     value codes  [kv_heads][head_dim / 2]
 *     key scales   [kv_heads][head_dim / 32]
 *     value scales [kv_heads][head_dim / 32]
 * = kv_heads * head_dim * 17 / 16 bytes, contiguous, so that a selected token
 * is one run of bytes. A token's slot is page * page_size + place in the
 * page.
 *
 * Array arguments are DEVICE pointers on the current HIP device, owned by the
 * caller; structs are HOST pointers read during the call. Work is enqueued on
 * `stream` (a hipStream_t as void*); nothing is allocated and nothing
 * synchronises, so every call may be captured into a HIP graph. Errors are
 * reported before anything is enqueued.
 */
#ifndef GVR_KV4_H
#define GVR_KV4_H

#include <stddef.h>
#include <stdint.h>

#include "gvr_rotary.h"
#include "gvr_topk.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gvr_kv4_cache {
    uint8_t* data;       /* 16-byte aligned */
    int64_t pages;       /* pages * page_size <= 2^31 - 16 */
    int32_t page_size;   /* tokens: a power of two, 1 .. 65536 */
    int32_t kv_heads;    /* 1 .. 1024 */
    int32_t head_dim;    /* 64, 128 or 256 */
    int32_t reserved;    /* 0 */
} gvr_kv4_cache;

/* Bytes of a token's record, or -1 for unsupported heads or head_dim. */
int64_t gvr_kv4_record_bytes(int32_t kv_heads, int32_t head_dim);

/* Write T tokens: k and v [T][kv_heads][head_dim] (gvr_dtype, any strides)
 * into slots [T] int64; a slot outside [0, pages * page_size) is skipped (-1
 * marks padding). Two tokens of one call must not name the same slot. With
 * `cs` the keys are rotated at positions [T] int32 first (gvr_rotary.h; a
 * position outside the table makes NaN blocks), in float32 and not rounded
 * before they are quantised. cs NULL: no rotation, positions is not read.
 * Errors: GVR_ERR_INVALID_ARG (a NULL pointer with T > 0, a bad cache, dtype,
 * rot > head_dim or flag), GVR_ERR_TOO_LONG (T > 2^31 - 16 or too many
 * slots), GVR_ERR_HIP. T == 0 is a no-op. */
gvr_status gvr_kv4_append(const gvr_kv4_cache* cache, const gvr_heads* k, const gvr_heads* v, int32_t dtype, int64_t T,
                          const int64_t* slots, const int32_t* positions, const gvr_rope_cs* cs, void* stream);

/* Read T tokens back: k and v [T][kv_heads][head_dim] of type `dtype` receive
 * the values that the records at slots [T] stand for (exact in bfloat16 and
 * float32, where only a code of 2^128 overflows; rounded in float16); zeros
 * for a slot outside the cache. Either of k and v may be NULL. Errors as gvr_kv4_append. */
gvr_status gvr_kv4_read(const gvr_kv4_cache* cache, const gvr_heads* k, const gvr_heads* v, int32_t dtype, int64_t T,
                        const int64_t* slots, void* stream);

/* Attention of T query tokens over the cache. Sequence b (of `sequences`)
 * holds ctx_len[b] tokens (clamped to [0, table_width * page_size]); token t
 * is place t % page_size of page block_table[b][t / page_size]; a page number
 * outside [0, pages) makes its tokens invisible. The sequence's query tokens
 * are rows q_start[b] .. q_start[b+1]-1 of q (n_q of them, at most max_q are
 * served, and rows that are not served are not written; the launch is planned
 * for max_q rows of every sequence, so it should be no more than their most;
 * q_start NULL: T / sequences each). The queries are the last tokens
 * of the context: with `causal`, query i sees t <= ctx_len[b] - n_q + i, else
 * every t < ctx_len[b]. With `selection` [T][K] int32, query row r attends
 * only to the tokens that its list names and the rule above allows (entries
 * below 0 or above the last allowed one are ignored; one named twice counts
 * twice): the out_idx of gvr_topk as it is. KV head h serves the query heads
 * [h G, (h+1) G), G = q_heads / kv_heads.
 *     out = sum_t w_t v_t,  w = softmax over visible t of scale * (q . k_t)
 *     lse = log sum_t exp(scale * (q . k_t))   (natural log; -inf if none)
 * A query that sees no token gives out = 0. Masked tokens are never part of a
 * result, whatever their records hold (NaN blocks and infinities included).
 *
 * Numerics: the stored keys enter the matrix cores as they are, the queries as
 * sums of two 8-bit numbers (three for float16) with a common scale per 32
 * elements: exact down to 2^-13 (2^-14) of the block's largest magnitude and
 * off by at most 2^-21 (2^-25) of it below. A score sums in float32 and is off
 * by about 2^-16 of scale * sum |q k|; in bfloat16 scale * (q . k) must stay
 * below 2^30 in magnitude. The softmax's maximum and sum are float32; the
 * weights, relative to the largest, and the stored values (exact; with float16
 * queries they must be below 65520, and are rounded to multiples of 2^-24) enter
 * the second product in the queries' type (float16: a weight is off by at most
 * 2^-40 of the largest beside its rounding); it sums in float32, and the result
 * is rounded once: about 0.0017 relative error in bfloat16, of which 0.0016 is
 * that last rounding. Rounding depends on how the context is split (the
 * workspace below, and with several sequences their lengths), never on timing:
 * the same call gives the same bits. */
typedef struct gvr_kv4_attention_args {
    const void* q;               /* [T][q_heads][head_dim], 16-byte aligned rows */
    int64_t q_token_stride;      /* elements, multiples of 8 */
    int64_t q_head_stride;
    void* out;                   /* [T][q_heads][head_dim] contiguous, 16-byte aligned */
    float* lse;                  /* [T][q_heads] or NULL */
    const int32_t* block_table;  /* [sequences][table_width] */
    const int32_t* ctx_len;      /* [sequences] */
    const int32_t* q_start;      /* [sequences + 1] or NULL */
    const int32_t* selection;    /* [T][K] or NULL */
    int64_t T;
    int64_t table_width;         /* pages per sequence */
    int32_t sequences;
    int32_t max_q;               /* most query tokens of a sequence (with q_start; else not read) */
    int32_t q_heads;             /* a multiple of kv_heads, at most 128 * kv_heads */
    int32_t K;                   /* selection entries per row */
    int32_t dtype;               /* GVR_BF16 or GVR_F16 */
    int32_t causal;              /* 0 or 1 */
    float scale;
    int32_t reserved;            /* 0 */
} gvr_kv4_attention_args;

/* Bytes of workspace with which the call splits long contexts over the whole
 * device (0: it does not split). Pointers in `args` are not read and may be
 * NULL, except that selection and q_start count as given when not NULL. */
gvr_status gvr_kv4_attention_workspace(const gvr_kv4_cache* cache, const gvr_kv4_attention_args* args, size_t* bytes);

/* The attention. workspace: 16-byte aligned device memory of ws_bytes, used
 * by this call only while it runs (no clearing needed); less than the call
 * asks for lowers the split, NULL with 0 bytes runs unsplit.
 * Errors: GVR_ERR_INVALID_ARG (a NULL or misaligned required pointer, bad
 * sizes, heads, dtype, or a workspace NULL with bytes), GVR_ERR_TOO_LONG
 * (table_width * page_size or T above 2^31 - 16, or a grid of 2^32 threads or
 * more), GVR_ERR_HIP.
 * T == 0, sequences == 0 or max_q == 0 with q_start is a no-op. */
gvr_status gvr_kv4_attention(const gvr_kv4_cache* cache, const gvr_kv4_attention_args* args, void* workspace,
                             size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GVR_KV4_H */
