// kv4_cache.hip -- tokens into and out of the paged 4-bit cache, behind
// include/gvr_kv4.h.
//
// Append: one thread takes eight elements of a head's key and of its value;
// the four lanes of a quad hold a block of 32, so the block's largest
// magnitude is two quad exchanges, the scale its exponent, and gfx950's
// conversion packs two codes per instruction (round to nearest even,
// saturating: what the format asks). A thread serves heads_each heads of its
// token in turn with the same cosines. Bound by HBM: a key and value element
// is read once and 4.25 bits of each written (16384 tokens of 8 heads of 128
// with rotation, appended and read back from HBM: 43 us = 4.2 TB/s; the append
// alone, what it reads still in the caches, 19, the reading 15); one token: 4 us
// each, the launch and four or five loads one after the other (slot, position,
// table row, key, in the half layout its partner). Unaligned rows load element by
// element (that append: 43 us against 18).

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "gvr_kv4.h"
#include "elem_ops.h"
#include "kv4_plan.h"
#include "wave_ops.h"

namespace {

using namespace gvr_elem;
using gvr_rot::kBlock;

struct TokenParams {
    uint8_t* cache;
    void* k;
    void* v;
    const int64_t* slots;
    const int32_t* positions;
    const float* cs;
    int64_t kt, kh, vt, vh;   // strides in elements
    int64_t n_slots, n_pos, T, tokens, record;
    int32_t H, D, rot, head_groups, heads_each;
    bool inter;
};

// Where the parts of head h's record start, for the eight elements at e.
struct Place {
    int64_t codes, scale;
};
DEV Place place(const TokenParams& p, int64_t slot, bool value, int h, int e) {
    const int64_t at = slot * p.record + (value ? (int64_t)p.H * p.D / 2 : 0);
    Place r;
    r.codes = at + ((int64_t)h * p.D + e) / 2;
    r.scale = slot * p.record + (int64_t)p.H * p.D + ((value ? (int64_t)p.H * p.D : 0) + (int64_t)h * p.D + e) / 32;
    return r;
}

struct Item {
    int64_t t;
    int hg, e;   // head group, first of the eight elements
    bool live;
};
DEV Item item_of(const TokenParams& p) {
    const uint32_t idx = blockIdx.x * (uint32_t)kBlock + threadIdx.x;
    const uint32_t per_head = (uint32_t)p.D / 8, per = (uint32_t)p.head_groups * per_head;
    const uint32_t t = idx / per, r = idx - t * per;
    Item it;
    it.hg = (int)(r / per_head);
    it.e = 8 * (int)(r % per_head);
    it.t = (int64_t)blockIdx.y * p.tokens + t;
    it.live = (int64_t)t < p.tokens && it.t < p.T;
    return it;
}

// The scale byte of a block from the bits of its largest magnitude: the least
// power of two that keeps it within 7 times the scale (1.75 * 2^2), not under
// 2^-126; 255 (NaN) for infinities and NaN.
DEV uint32_t scale_byte(uint32_t bits) {
    const int e = (int)(bits >> 23);
    const int b = e - 2 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e == 255 ? 255u : (uint32_t)max(b, 1);
}

// Quantise the quad's block and write this lane's eight codes and, from the
// quad's first lane, the scale.
DEV void put(const TokenParams& p, const Place& at, f8 x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    m = max(m, (uint32_t)gvr_dev::dpp_i<gvr_dev::kQuadSwap1>(0, (int)m));
    m = max(m, (uint32_t)gvr_dev::dpp_i<gvr_dev::kQuadSwap2>(0, (int)m));
    const uint32_t byte = scale_byte(m);
    const float scale = __uint_as_float(byte << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    *reinterpret_cast<uint32_t*>(p.cache + at.codes) = codes;
    if ((threadIdx.x & 3) == 0) p.cache[at.scale] = (uint8_t)byte;
}

enum { kNoTurn, kHalf, kInter, kAny };   // rotations; kAny also serves unaligned rows

template <class E, int MODE>
__global__ __launch_bounds__(kBlock) void append_kernel(TokenParams p) {
    constexpr bool WIDE = MODE != kAny;
    const Item it = item_of(p);
    if (!it.live) return;
    const int64_t slot = p.slots[it.t];
    if (slot < 0 || slot >= p.n_slots) return;
    const int half = p.rot / 2;
    const bool turn = MODE != kNoTurn && it.e < p.rot;
    const float* row = nullptr;
    if (turn) {
        const int32_t pos = p.positions[it.t];
        if (pos >= 0 && pos < p.n_pos) row = p.cs + (int64_t)pos * p.rot;
    }
    // half layout: this run's partners and pairs
    const bool second = MODE == kHalf && it.e >= half;
    const int other = second ? it.e - half : it.e + half;
    float c[8], s[8];
    if (turn) {
        if constexpr (MODE == kHalf) load_cs<8, true>(row, second ? other : it.e, c, s);
        if constexpr (MODE == kInter) {
            float c4[4], s4[4];
            load_cs<4, true>(row, it.e / 2, c4, s4);
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = c4[i], s[i] = s4[i];
        }
    }
    const E* k = static_cast<const E*>(p.k) + it.t * p.kt;
    const E* v = static_cast<const E*>(p.v) + it.t * p.vt;
    for (int j = 0; j < p.heads_each; ++j) {
        const int h = j * p.head_groups + it.hg;
        if (h >= p.H) break;
        const E* kp = k + h * p.kh;
        f8 x = load8<WIDE>(kp + it.e);
        const f8 y = load8<WIDE>(v + h * p.vh + it.e);
        if (turn) {
            if constexpr (MODE == kHalf) {
                const f8 o = load8<true>(kp + other);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = second ? turn_b(o[i], x[i], c[i], s[i]) : turn_a(x[i], o[i], c[i], s[i]);
            } else if constexpr (MODE == kInter) {
                const f8 o = x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = turn_a(o[2 * i], o[2 * i + 1], c[i], s[i]);
                    x[2 * i + 1] = turn_b(o[2 * i], o[2 * i + 1], c[i], s[i]);
                }
            } else if constexpr (MODE == kAny) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = it.e + i;
                    if (e < p.rot) {
                        const bool b = p.inter ? e & 1 : e >= half;
                        const int pair = p.inter ? e / 2 : (b ? e - half : e);
                        const float o = (float)kp[p.inter ? e ^ 1 : (b ? e - half : e + half)];
                        float ci[1], si[1];
                        load_cs<1, false>(row, pair, ci, si);
                        x[i] = b ? turn_b(o, x[i], ci[0], si[0]) : turn_a(x[i], o, ci[0], si[0]);
                    }
                }
            }
        }
        put(p, place(p, slot, false, h, it.e), x);
        put(p, place(p, slot, true, h, it.e), y);
    }
}

DEV f8 get(const TokenParams& p, const Place& at) {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(p.cache + at.codes);
    const float scale = __uint_as_float((uint32_t)p.cache[at.scale] << 23);
    f8 x;
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
    const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
    const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
    return x;
}

template <class E, bool WIDE>
__global__ __launch_bounds__(kBlock) void read_kernel(TokenParams p) {
    const Item it = item_of(p);
    if (!it.live) return;
    const int64_t slot = p.slots[it.t];
    const bool held = slot >= 0 && slot < p.n_slots;
    for (int j = 0; j < p.heads_each; ++j) {
        const int h = j * p.head_groups + it.hg;
        if (h >= p.H) break;
        f8 x = {0, 0, 0, 0, 0, 0, 0, 0}, y = x;
        if (held) {
            if (p.k) x = get(p, place(p, slot, false, h, it.e));
            if (p.v) y = get(p, place(p, slot, true, h, it.e));
        }
        if (p.k) store8<WIDE>(static_cast<E*>(p.k) + it.t * p.kt + h * p.kh + it.e, x);
        if (p.v) store8<WIDE>(static_cast<E*>(p.v) + it.t * p.vt + h * p.vh + it.e, y);
    }
}

// What both calls check and fill in; *go: there is something to launch.
gvr_status token_params(const gvr_kv4_cache* cache, const gvr_heads* k, const gvr_heads* v, int32_t dtype, int64_t T,
                        const int64_t* slots, TokenParams* p, gvr_rot::Launch* l) {
    const int size = gvr_rot::dtype_size(dtype);
    if (size == 0 || T < 0) return GVR_ERR_INVALID_ARG;
    const gvr_status st = gvr_kv4::check_cache(cache, T > 0);
    if (st != GVR_OK) return st;
    if (T > gvr_rot::kMaxCount) return GVR_ERR_TOO_LONG;
    if (T > 0 && !slots) return GVR_ERR_INVALID_ARG;
    for (const gvr_heads* h : {k, v})
        if (h && ((uintptr_t)h->data & (size - 1))) return GVR_ERR_INVALID_ARG;
    p->cache = cache->data;
    p->k = k ? k->data : nullptr;
    p->v = v ? v->data : nullptr;
    p->kt = k ? k->token_stride : 0, p->kh = k ? k->head_stride : 0;
    p->vt = v ? v->token_stride : 0, p->vh = v ? v->head_stride : 0;
    p->slots = slots;
    p->n_slots = cache->pages * cache->page_size;
    p->record = gvr_kv4::record_bytes(cache->kv_heads, cache->head_dim);
    p->T = T;
    p->H = cache->kv_heads, p->D = cache->head_dim;
    p->positions = nullptr, p->cs = nullptr, p->n_pos = 0, p->rot = 0, p->inter = false;
    if (T > 0) {
        *l = gvr_rot::plan_items(T, p->H, p->D / 8, 2);
        p->heads_each = l->heads_each;
        p->head_groups = l->head_groups;
        p->tokens = l->tokens;
        if (l->rows > gvr_rot::kMaxRows) return GVR_ERR_TOO_LONG;
    }
    return GVR_OK;
}

template <class E>
gvr_status launch_append(const TokenParams& p, const gvr_rot::Launch& l, int mode, void* stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks, (unsigned)l.rows), dim3(kBlock), 0, (hipStream_t)stream, p);
    };
    mode == kNoTurn ? go(append_kernel<E, kNoTurn>)
    : mode == kHalf ? go(append_kernel<E, kHalf>)
    : mode == kInter ? go(append_kernel<E, kInter>) : go(append_kernel<E, kAny>);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

template <class E>
gvr_status launch_read(const TokenParams& p, const gvr_rot::Launch& l, bool wide, void* stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks, (unsigned)l.rows), dim3(kBlock), 0, (hipStream_t)stream, p);
    };
    wide ? go(read_kernel<E, true>) : go(read_kernel<E, false>);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // namespace

extern "C" {

int64_t gvr_kv4_record_bytes(int32_t kv_heads, int32_t head_dim) { return gvr_kv4::record_bytes(kv_heads, head_dim); }

gvr_status gvr_kv4_append(const gvr_kv4_cache* cache, const gvr_heads* k, const gvr_heads* v, int32_t dtype, int64_t T,
                          const int64_t* slots, const int32_t* positions, const gvr_rope_cs* cs, void* stream) {
    if (!k || !v) return GVR_ERR_INVALID_ARG;
    TokenParams p;
    gvr_rot::Launch l;
    const gvr_status st = token_params(cache, k, v, dtype, T, slots, &p, &l);
    if (st != GVR_OK) return st;
    if (cs) {
        const gvr_status s = gvr_rot::check_cs(*cs, p.D, GVR_ROPE_INTERLEAVED);
        if (s != GVR_OK) return s;
        if (T > 0 && !positions) return GVR_ERR_INVALID_ARG;
    }
    if (T == 0) return GVR_OK;
    if (!p.k || !p.v) return GVR_ERR_INVALID_ARG;
    const int size = gvr_rot::dtype_size(dtype);
    const bool wide = gvr_rot::wide_rows(*k, size) && gvr_rot::wide_rows(*v, size);
    int mode = wide ? kNoTurn : kAny;
    if (cs) {
        p.positions = positions;
        p.cs = cs->data, p.n_pos = cs->positions, p.rot = cs->rot;
        p.inter = cs->flags & GVR_ROPE_INTERLEAVED;
        if (!wide || !gvr_rot::wide_cs(*cs))
            mode = kAny;
        else if (p.inter)
            mode = p.rot % 8 == 0 ? kInter : kAny;
        else
            mode = p.rot % 16 == 0 ? kHalf : kAny;
    }
    return dtype == GVR_BF16 ? launch_append<__bf16>(p, l, mode, stream)
           : dtype == GVR_F16 ? launch_append<_Float16>(p, l, mode, stream)
                              : launch_append<float>(p, l, mode, stream);
}

gvr_status gvr_kv4_read(const gvr_kv4_cache* cache, const gvr_heads* k, const gvr_heads* v, int32_t dtype, int64_t T,
                        const int64_t* slots, void* stream) {
    TokenParams p;
    gvr_rot::Launch l;
    const gvr_status st = token_params(cache, k, v, dtype, T, slots, &p, &l);
    if (st != GVR_OK) return st;
    if (T == 0 || (!p.k && !p.v)) return GVR_OK;
    const int size = gvr_rot::dtype_size(dtype);
    const bool wide = (!p.k || gvr_rot::wide_rows(*k, size)) && (!p.v || gvr_rot::wide_rows(*v, size));
    return dtype == GVR_BF16 ? launch_read<__bf16>(p, l, wide, stream)
           : dtype == GVR_F16 ? launch_read<_Float16>(p, l, wide, stream)
                              : launch_read<float>(p, l, wide, stream);
}

}  // extern "C"
