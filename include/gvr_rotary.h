/*
 * gvr_rotary.h -- rotary positions on MI355X (gfx950): the table of cosines
 * and sines of RoPE / YaRN-scaled positions, and the rotation of query or key
 * heads by it (and of gradients, by its transpose).
 *
 * A head's first R elements are R/2 pairs (a_i, b_i). At position p pair i is
 * turned by the angle p theta'_i (the angles of gvr_rope_prior.h) and scaled
 * by `gain` (YaRN's attention factor; 1 = none), both held in the table:
 *     c = gain cos(p theta'_i),  s = gain sin(p theta'_i)
 *     a'_i = a_i c - b_i s,      b'_i = b_i c + a_i s
 * Pairs: "half" layout a_i = x[i], b_i = x[i + R/2]; "interleaved" layout
 * a_i = x[2i], b_i = x[2i+1]. Elements R .. D-1 are copied. The transposed
 * rotation (s -> -s) maps the gradient of the output to that of the input,
 * and undoes the rotation when gain = 1.
 *
 * Rounding: the products and the sum are float32, each rounded once (no
 * fused multiply-add), and the result is rounded once to the tensor's type.
 *
 * Array arguments are DEVICE pointers on the current HIP device, owned by the
 * caller; structs are HOST pointers read during the call. Work is enqueued on
 * `stream` (a hipStream_t as void*) as one kernel; nothing is allocated and
 * nothing synchronises, so the calls may be captured into a HIP graph.
 */
#ifndef GVR_ROTARY_H
#define GVR_ROTARY_H

#include <stdint.h>

#include "gvr_rope_prior.h"
#include "gvr_topk.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { GVR_BF16 = 0, GVR_F16 = 1, GVR_F32 = 2 } gvr_dtype;

/* Heads of T tokens: element (t, h, d) is data[t token_stride + h head_stride
 * + d], strides in elements. */
typedef struct gvr_heads {
    void* data;
    int64_t token_stride;
    int64_t head_stride;
} gvr_heads;

/* Cosines and sines: cs[p][i] = {c, s}, p < positions, i < R/2, float32. */
typedef struct gvr_rope_cs {
    const float* data;   /* [positions][rot / 2][2], 8-byte aligned */
    int64_t positions;
    int32_t rot;         /* R: even, 2 .. 512 */
    int32_t flags;       /* GVR_ROPE_* */
} gvr_rope_cs;
enum {
    GVR_ROPE_INTERLEAVED = 1,   /* pairs (2i, 2i+1) instead of (i, i + R/2) */
    GVR_ROPE_TRANSPOSED = 2     /* the gradient's rotation (s -> -s); gvr_rope_rotate only */
};

/* Fill table [n][d_rope / 2][2] float32 with gain * cos, gain * sin of the
 * positions 0 .. n-1; angles and functions are float64, rounded once.
 * Errors: GVR_ERR_INVALID_ARG (n < 0, bad params, gain not finite, table NULL
 * with n > 0 or not 8-byte aligned), GVR_ERR_TOO_LONG (n > 2^31 - 16),
 * GVR_ERR_HIP. */
gvr_status gvr_rope_table(int64_t n, const gvr_rope_params* params, double gain, float* table, void* stream);

/* out = x rotated. x and out: [T][H][D] with their own strides, both of type
 * `dtype`; out may be x itself (same data and strides), else they must not
 * overlap. positions [T] int32: a position outside [0, cs->positions) turns
 * its token's rotated elements into NaN.
 * Supported: 1 <= D <= 1024, rot <= D. Any strides and element alignment
 * (16-byte aligned rows with rot and D - rot multiples of 16 take the wide
 * loads).
 * Errors: GVR_ERR_INVALID_ARG (a NULL or misaligned pointer, T < 0, H < 0, a
 * bad D, rot, dtype, flag or positions count), GVR_ERR_TOO_LONG (T above
 * 2^31 - 16 or H above 2^20), GVR_ERR_HIP. T == 0 or H == 0 is a no-op. */
gvr_status gvr_rope_rotate(const gvr_heads* x, const gvr_heads* out, int32_t dtype, int64_t T, int32_t H, int32_t D,
                           const int32_t* positions, const gvr_rope_cs* cs, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GVR_ROTARY_H */
