// rotary.hip -- the cosine / sine table of RoPE / YaRN positions and the
// rotation of heads by it, behind include/gvr_rotary.h.
//
// Rotation: one thread turns eight pairs of a head (half layout: eight
// elements of the first half and their eight partners; interleaved: sixteen
// consecutive ones) or copies sixteen elements behind the rotary ones, for
// heads_each heads of one token in turn, so that the eight cosines and sines
// are read once for all of them. Bound by HBM: each element is read once and
// written once (8192 tokens of 32 heads of 128 in bfloat16, 138 MB with the
// table: 27.9 us = 4.95 TB/s, where a copy of 1 GB reaches 4.8); smaller calls by
// the launch and three loads one after the other, position, table row and only
// then the elements (35 MB of float32: 10.5 us, 7.3 at the copy's rate; a decode
// step's 128 x 64 heads: 3.9 us).
// Rows that are not 16-byte aligned, or whose rotary part is no multiple of 16,
// take a kernel that loads element by element (8192 x 64 x 128 in bfloat16:
// 42 us wide, 55 us by element; 1024 x 32: 4.8 and 6.2).

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "gvr_rotary.h"
#include "elem_ops.h"
#include "rotary_plan.h"
#include "yarn.h"

namespace {

using namespace gvr_elem;
using gvr_rot::kBlock;

struct RotParams {
    const void* x;
    void* out;
    const int32_t* positions;
    const float* cs;
    int64_t xt, xh, ot, oh;   // strides in elements
    int64_t n_pos, T, tokens;
    int32_t H, D, rot, per_head, head_groups, heads_each;
    float sign;               // of s: -1 for the transposed rotation
};

struct Item {
    int64_t t;
    int hg, c;
    bool live;
};
DEV Item item_of(const RotParams& p) {
    const uint32_t idx = blockIdx.x * (uint32_t)kBlock + threadIdx.x;
    const uint32_t per = (uint32_t)p.head_groups * (uint32_t)p.per_head;
    const uint32_t t = idx / per, r = idx - t * per;
    Item it;
    it.hg = (int)(r / (uint32_t)p.per_head);
    it.c = (int)(r - (uint32_t)it.hg * (uint32_t)p.per_head);
    it.t = (int64_t)blockIdx.y * p.tokens + t;
    it.live = (int64_t)t < p.tokens && it.t < p.T;
    return it;
}
DEV const float* cs_row(const RotParams& p, int64_t t) {
    const int32_t pos = p.positions[t];
    return pos >= 0 && pos < p.n_pos ? p.cs + (int64_t)pos * p.rot : nullptr;
}

template <class E, bool INTER>
__global__ __launch_bounds__(kBlock) void rotate_wide_kernel(RotParams p) {
    const Item it = item_of(p);
    if (!it.live) return;
    const int chunks = p.rot / 16;   // of eight pairs
    const bool turn = it.c < chunks;
    // the sixteen elements: two runs of eight
    const int e0 = turn ? (INTER ? 16 * it.c : 8 * it.c) : p.rot + 16 * (it.c - chunks);
    const int e1 = turn && !INTER ? e0 + p.rot / 2 : e0 + 8;
    float c[8], s[8];
    if (turn) load_cs<8, true>(cs_row(p, it.t), 8 * it.c, c, s);
    const E* x = static_cast<const E*>(p.x) + it.t * p.xt;
    E* out = static_cast<E*>(p.out) + it.t * p.ot;
#pragma unroll 2
    for (int j = 0; j < p.heads_each; ++j) {
        const int h = j * p.head_groups + it.hg;
        if (h >= p.H) break;
        f8 u = load8<true>(x + h * p.xh + e0), v = load8<true>(x + h * p.xh + e1);
        if (turn) {
            if constexpr (INTER) {
                f8 y0, y1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y0[2 * i] = turn_a(u[2 * i], u[2 * i + 1], c[i], p.sign * s[i]);
                    y0[2 * i + 1] = turn_b(u[2 * i], u[2 * i + 1], c[i], p.sign * s[i]);
                    y1[2 * i] = turn_a(v[2 * i], v[2 * i + 1], c[4 + i], p.sign * s[4 + i]);
                    y1[2 * i + 1] = turn_b(v[2 * i], v[2 * i + 1], c[4 + i], p.sign * s[4 + i]);
                }
                u = y0, v = y1;
            } else {
                f8 y0, y1;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    y0[i] = turn_a(u[i], v[i], c[i], p.sign * s[i]);
                    y1[i] = turn_b(u[i], v[i], c[i], p.sign * s[i]);
                }
                u = y0, v = y1;
            }
        }
        store8<true>(out + h * p.oh + e0, u);
        store8<true>(out + h * p.oh + e1, v);
    }
}

// Any sizes, strides and alignment: one thread per pair, then per copied element.
template <class E, bool INTER>
__global__ __launch_bounds__(kBlock) void rotate_any_kernel(RotParams p) {
    const Item it = item_of(p);
    if (!it.live) return;
    const int half = p.rot / 2;
    const bool turn = it.c < half;
    const int e0 = turn ? (INTER ? 2 * it.c : it.c) : half + it.c;
    const int e1 = INTER ? e0 + 1 : e0 + half;
    float c[1], s[1];
    if (turn) load_cs<1, false>(cs_row(p, it.t), it.c, c, s);
    const E* x = static_cast<const E*>(p.x) + it.t * p.xt;
    E* out = static_cast<E*>(p.out) + it.t * p.ot;
    for (int j = 0; j < p.heads_each; ++j) {
        const int h = j * p.head_groups + it.hg;
        if (h >= p.H) break;
        if (turn) {
            const float a = (float)x[h * p.xh + e0], b = (float)x[h * p.xh + e1];
            out[h * p.oh + e0] = (E)turn_a(a, b, c[0], p.sign * s[0]);
            out[h * p.oh + e1] = (E)turn_b(a, b, c[0], p.sign * s[0]);
        } else {
            out[h * p.oh + e0] = x[h * p.xh + e0];
        }
    }
}

// Table: a workgroup's first R/2 threads hold the angles in LDS, then each
// thread makes pairs of `rows` positions. Bound by the float64 functions: 131072
// positions of 64 pairs (67 MB) 31.5 us = 2.1 TB/s, 8192 of 32 pairs 9.5 us.
__global__ __launch_bounds__(gvr_yarn::kMaxPairs) void rope_table_kernel(int64_t n, int rows, gvr_yarn::RopeArgs a,
                                                                         double gain, float* __restrict__ table) {
    __shared__ double th[gvr_yarn::kMaxPairs];
    const int half = a.d / 2;
    if ((int)threadIdx.x < half) th[threadIdx.x] = gvr_yarn::yarn_angle(threadIdx.x, a);
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * rows;
    const int items = (int)(n - p0 < rows ? n - p0 : rows) * half;
    for (int i = threadIdx.x; i < items; i += gvr_yarn::kMaxPairs) {
        const int64_t pos = p0 + i / half;
        const int pair = i % half;
        double s, c;
        sincos((double)pos * th[pair], &s, &c);
        float2 v;
        v.x = (float)(gain * c), v.y = (float)(gain * s);
        reinterpret_cast<float2*>(table)[pos * half + pair] = v;
    }
}

template <class E>
gvr_status launch_rotate(RotParams p, bool wide, bool inter, void* stream) {
    p.per_head = wide ? p.D / 16 : p.rot / 2 + p.D - p.rot;
    const gvr_rot::Launch l = gvr_rot::plan_items(p.T, p.H, p.per_head, 2);
    p.heads_each = l.heads_each;
    p.head_groups = l.head_groups;
    p.tokens = l.tokens;
    if (l.rows > gvr_rot::kMaxRows) return GVR_ERR_TOO_LONG;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks, (unsigned)l.rows), dim3(kBlock), 0, (hipStream_t)stream, p);
    };
    if (wide)
        inter ? go(rotate_wide_kernel<E, true>) : go(rotate_wide_kernel<E, false>);
    else
        inter ? go(rotate_any_kernel<E, true>) : go(rotate_any_kernel<E, false>);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // namespace

extern "C" {

gvr_status gvr_rope_table(int64_t n, const gvr_rope_params* params, double gain, float* table, void* stream) {
    gvr_yarn::RopeArgs a;
    const gvr_status st = gvr_yarn::read_params(params, &a);
    if (st != GVR_OK) return st;
    if (n < 0 || !isfinite(gain) || (n > 0 && !table) || ((uintptr_t)table & 7)) return GVR_ERR_INVALID_ARG;
    if (n > gvr_rot::kMaxCount) return GVR_ERR_TOO_LONG;
    if (n == 0) return GVR_OK;
    const int rows = gvr_rot::table_rows(n);
    hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + rows - 1) / rows)), dim3(gvr_yarn::kMaxPairs), 0,
                       (hipStream_t)stream, n, rows, a, gain, table);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

gvr_status gvr_rope_rotate(const gvr_heads* x, const gvr_heads* out, int32_t dtype, int64_t T, int32_t H, int32_t D,
                           const int32_t* positions, const gvr_rope_cs* cs, void* stream) {
    const int size = gvr_rot::dtype_size(dtype);
    if (!x || !out || !cs || size == 0 || T < 0 || H < 0 || D < 1 || D > 1024) return GVR_ERR_INVALID_ARG;
    gvr_status st = gvr_rot::check_cs(*cs, D, GVR_ROPE_INTERLEAVED | GVR_ROPE_TRANSPOSED);
    if (st != GVR_OK) return st;
    if (T > gvr_rot::kMaxCount || H > (1 << 20)) return GVR_ERR_TOO_LONG;
    if (T == 0 || H == 0) return GVR_OK;
    if (!x->data || !out->data || !positions) return GVR_ERR_INVALID_ARG;
    if (((uintptr_t)x->data | (uintptr_t)out->data) & (size - 1)) return GVR_ERR_INVALID_ARG;
    RotParams p;
    p.x = x->data, p.xt = x->token_stride, p.xh = x->head_stride;
    p.out = out->data, p.ot = out->token_stride, p.oh = out->head_stride;
    p.positions = positions;
    p.cs = cs->data, p.n_pos = cs->positions, p.rot = cs->rot;
    p.T = T, p.H = H, p.D = D;
    p.sign = cs->flags & GVR_ROPE_TRANSPOSED ? -1.f : 1.f;
    const bool inter = cs->flags & GVR_ROPE_INTERLEAVED;
    const bool wide = cs->rot % 16 == 0 && D % 16 == 0 && gvr_rot::wide_cs(*cs) && gvr_rot::wide_rows(*x, size) &&
                      gvr_rot::wide_rows(*out, size);
    return dtype == GVR_BF16 ? launch_rotate<__bf16>(p, wide, inter, stream)
           : dtype == GVR_F16 ? launch_rotate<_Float16>(p, wide, inter, stream)
                              : launch_rotate<float>(p, wide, inter, stream);
}

}  // extern "C"
