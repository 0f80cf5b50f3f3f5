// kv4_attention.hip -- attention over the paged 4-bit cache, behind
// include/gvr_kv4.h.
//
// One wave serves 16 query rows (the query heads of one KV head, of one or
// more query tokens of a sequence) over a chunk of the context, 32 tokens a
// step, on the 16-bit matrix cores:
//     S^T [tokens][rows] = K Q^T,   P = exp2(S - m),   O^T [dims][rows] += V^T P^T
// Lane l holds column l % 16 (its query row) and quarter l / 16. The order of
// the dimensions inside the first product and of the tokens inside the second
// is free, and is chosen so that nothing moves between lanes:
//   - K: a lane takes D / 4 consecutive dimensions of one token per 16, one
//     load of D / 8 bytes of codes that share one scale (D = 256: two);
//   - the scores that come out sit in the lane that feeds them, as weights, to
//     the second product: tokens 4 q + i of both halves of the step;
//   - V: for those tokens a lane takes D / 16 consecutive dimensions, and the
//     n-th of them goes to the n-th matrix step.
// gfx950's conversion turns two codes and their scale into two 16-bit floats
// in one instruction; the values of two tokens are then paired by byte
// permutes. Running maximum and sum are float32 per row; chunks of one
// context are joined by a second kernel from float32 partial results.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "gvr_kv4.h"
#include "kv4_plan.h"
#include "wave_ops.h"

namespace {

using gvr_kv4::kRows;
using gvr_kv4::kStep;
using gvr_kv4::kWaves;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
template <class E> struct Vec { typedef E x8 __attribute__((ext_vector_type(8))); typedef E x2 __attribute__((ext_vector_type(2))); };

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;

struct AttnParams {
    const uint8_t* cache;
    const void* q;
    void* out;
    float* lse;
    float* part_o;    // [T][q_heads][splits][D]
    float* part_ml;   // [T][q_heads][splits][2]: maximum (log2 domain), sum
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* q_start;
    const int32_t* selection;
    int64_t qt, qh;   // query strides
    int64_t table_width, pages, record, T, jobs;
    int32_t page_shift, kv_heads, q_heads, group, sequences, uniform_q, max_q, tiles, splits, chunk, K, causal;
    float scale2;     // scale * log2(e)
};

// Two codes (byte `sel` of w) times the scale as a packed pair.
template <class E>
DEV uint32_t unpack(uint32_t w, float scale, int sel) {
    typename Vec<E>::x2 v;
    if constexpr (sizeof(E) == 2 && __is_same(E, __bf16)) {
        v = sel == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
            : sel == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
            : sel == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    } else {
        v = sel == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)
            : sel == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)
            : sel == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)
                       : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
    }
    return __builtin_bit_cast(uint32_t, v);
}
template <class E>
DEV v4f mfma(v4u a, v4u b, v4f c) {
    typedef typename Vec<E>::x8 x8;
    if constexpr (__is_same(E, __bf16))
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}
template <class E>
DEV uint32_t pack2(float a, float b) {
    typename Vec<E>::x2 v;
    v[0] = (E)a, v[1] = (E)b;
    return __builtin_bit_cast(uint32_t, v);
}
DEV float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// NB bytes of codes at p as dwords (4-byte aligned; two bytes: 2-byte aligned).
template <int NB>
struct Codes {
    uint32_t w[NB / 4 ? NB / 4 : 1];
};
template <int NB>
DEV Codes<NB> load_codes(const uint8_t* p) {
    Codes<NB> c;
    if constexpr (NB == 2) {
        c.w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(NB / 4 > 4 ? 4 : NB / 4), aligned(4)));
#pragma unroll
        for (int i = 0; i < NB / 4; i += 4) {
            const vec v = *reinterpret_cast<const vec*>(p + 4 * i);
#pragma unroll
            for (int j = 0; j < (NB / 4 > 4 ? 4 : NB / 4); ++j) {
                if constexpr (NB == 4)
                    c.w[0] = v[0];
                else
                    c.w[i + j] = v[j];
            }
        }
    }
    return c;
}

// Sequence b's query tokens: rows q0 .. q0 + nq - 1 of q, the first `shown` served.
struct Rows {
    int64_t q0, nq;
    int shown;
};
DEV Rows rows_of(const AttnParams& p, int b) {
    Rows r;
    r.q0 = (int64_t)b * p.uniform_q, r.nq = p.uniform_q;
    if (p.q_start) {
        r.q0 = p.q_start[b];
        r.nq = (int64_t)p.q_start[b + 1] - r.q0;
        if (r.q0 < 0 || r.q0 > p.T) r.nq = 0;
        r.nq = min(r.nq, p.T - r.q0);
    }
    r.shown = (int)min(r.nq, (int64_t)p.max_q);
    return r;
}

template <class E, int D, bool SEL>
__global__ __launch_bounds__(kWaves * 64) void few_rows_kernel(AttnParams p) {
    constexpr int KS = D / 32;        // matrix steps of the first product
    constexpr int NT = D / 16;        // dimensions of V per lane = matrix steps of the second
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    // wave-uniform: head fastest (neighbouring waves read neighbouring parts of the records)
    int64_t job = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (job >= p.jobs) return;
    const int h = (int)(job % p.kv_heads);
    job /= p.kv_heads;
    const int tile = (int)(job % p.tiles);
    job /= p.tiles;
    const int split = (int)(job % p.splits);
    const int b = (int)(job / p.splits);

    const Rows rows = rows_of(p, b);
    const int64_t q0 = rows.q0, nq = rows.nq;
    const int shown = rows.shown;
    if (shown <= 0) return;
    const int64_t held = p.table_width << p.page_shift;
    const int ctx = (int)min((int64_t)max(p.ctx_len[b], 0), held);

    // this lane's query row
    int qi, qg;   // query token of the sequence, head of the group
    bool live;
    if constexpr (SEL) {
        const int per = (p.group + kRows - 1) / kRows;
        qi = tile / per;
        qg = (tile - qi * per) * kRows + col;
        live = qi < shown && qg < p.group;
        if (qi >= shown) return;
    } else {
        const int r = tile * kRows + col;
        qi = r / p.group;
        qg = r - qi * p.group;
        live = qi < shown;
        if ((tile * kRows) / p.group >= shown) return;
    }
    const int64_t row = q0 + qi;
    const int hq = h * p.group + qg;
    // last visible token of this row; of the wave's rows, the last row's is the largest
    const int last = live ? (p.causal ? (int)(ctx - nq + qi) : ctx - 1) : -1;
    int end;
    if constexpr (SEL) {
        end = p.K;
    } else {
        const int qi_last = min((tile * kRows + kRows - 1) / p.group, shown - 1);
        end = (int)max((int64_t)0, p.causal ? ctx - nq + qi_last + 1 : (int64_t)ctx);
    }
    const int64_t lo = (int64_t)split * p.chunk;
    const int begin = (int)min(lo, (int64_t)end), stop = (int)min(lo + p.chunk, (int64_t)end);

    // queries: for matrix step s the lane holds dimensions quarter * D / 4 + 8 s ..
    v4u qf[KS];
    {
        const uint16_t* qp = static_cast<const uint16_t*>(p.q) + (live ? row * p.qt + hq * p.qh : 0) + quarter * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const v4u v = *reinterpret_cast<const v4u*>(qp + 8 * s);
            qf[s] = live ? v : v4u{0, 0, 0, 0};
        }
    }
    const int64_t k_off = (int64_t)h * (D / 2) + quarter * (D / 8);
    const int64_t v_off = (int64_t)(p.kv_heads + h) * (D / 2) + col * (D / 32);
    const int64_t ks_off = (int64_t)p.kv_heads * D + h * (D / 32) + quarter * (D / 4) / 32;
    const int64_t vs_off = (int64_t)p.kv_heads * D + (p.kv_heads + h) * (D / 32) + col * (D / 16) / 32;
    const int32_t* table = p.block_table + (int64_t)b * p.table_width;
    const int32_t* list = SEL ? p.selection + row * p.K : nullptr;
    const int sel_last = SEL ? (p.causal ? (int)(ctx - nq + qi) : ctx - 1) : 0;   // the same for the wave's rows
    const int page_mask = (1 << p.page_shift) - 1;

    // last token that the wave's first row sees (all rows see what it sees)
    const int64_t first_last = p.causal ? ctx - nq + (tile * kRows) / p.group : (int64_t)ctx - 1;

    float m = -INFINITY, sum = 0.f;
    v4f o[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) o[n] = v4f{0.f, 0.f, 0.f, 0.f};

    for (int t0 = begin; t0 < stop; t0 += kStep) {
        // slots of tokens t0 + lane % 32 (-1: not there)
        int slot = -1;
        {
            const int n = t0 + (lane & 31);
            int tok = n;
            bool there = n < stop;
            if constexpr (SEL) {
                if (there) tok = list[n];
                there = there && tok >= 0 && tok <= sel_last;
            }
            if (there) {
                const int page = table[tok >> p.page_shift];
                if (page >= 0 && page < p.pages) slot = (page << p.page_shift) + (tok & page_mask);
            }
        }
        const uint32_t there = (uint32_t)__ballot(slot >= 0);
        if (there == 0) continue;
        slot = max(slot, 0);
        v4f sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* rec = p.cache + (int64_t)__shfl(slot, 16 * t + col, 64) * p.record;
            const Codes<D / 8> kc = load_codes<D / 8>(rec + k_off);
            const float s0 = scale_of(rec[ks_off]);
            const float s1 = D == 256 ? scale_of(rec[ks_off + 1]) : s0;
            v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const float ss = D == 256 && s >= KS / 2 ? s1 : s0;
                const v4u a = {unpack<E>(kc.w[s], ss, 0), unpack<E>(kc.w[s], ss, 1), unpack<E>(kc.w[s], ss, 2),
                               unpack<E>(kc.w[s], ss, 3)};
                acc = mfma<E>(a, qf[s], acc);
            }
            sc[t] = acc;
        }
        // mask, running maximum
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = 16 * t + 4 * quarter + i;
                const bool see = ((there >> n) & 1) && (SEL ? live : t0 + n <= last);
                sc[t][i] = see ? sc[t][i] * p.scale2 : -INFINITY;
                top = fmaxf(top, sc[t][i]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m, top);
        const float base = m_new == -INFINITY ? 0.f : m_new;   // nothing seen so far: all weights are zero
        const float keep = exp2f(m - base);
        m = m_new;
        sum *= keep;
        v4u pf;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = exp2f(sc[t][i] - base);
                sum += w[i];
            }
            pf[2 * t] = pack2<E>(w[0], w[1]);
            pf[2 * t + 1] = pack2<E>(w[2], w[3]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n] *= keep;
        // values: a masked token's weight is zero, and its codes are taken as
        // zero too (a NaN block times zero would not be)
        uint32_t vw[8][D == 256 ? 2 : 1];
        float vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int n = 16 * (j >> 2) + 4 * quarter + (j & 3);
            const uint8_t* rec = p.cache + (int64_t)__shfl(slot, n, 64) * p.record;
            const Codes<D / 32> c = load_codes<D / 32>(rec + v_off);
            const bool see = (there >> n) & 1;
#pragma unroll
            for (int i = 0; i < (D == 256 ? 2 : 1); ++i) vw[j][i] = see ? c.w[i] : 0u;
            vs[j] = see ? scale_of(rec[vs_off]) : 1.f;
        }
        // Where the wave's rows see different tokens, a NaN value block must
        // not meet the zero weight of a row that does not see it: it is taken
        // out, and the rows that see it are found by a product of indicators.
        if (!SEL && t0 + kStep - 1 > first_last) {
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) bad |= __float_as_uint(vs[j]) == 0x7F800000u ? 1u << j : 0u;
            if (__ballot(bad != 0)) {
                v4u ind, seen;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    ind[j] = pack2<E>((bad >> (2 * j)) & 1 ? 1.f : 0.f, (bad >> (2 * j + 1)) & 1 ? 1.f : 0.f);
                    seen[j] = pack2<E>(sc[j >> 1][2 * (j & 1)] > -INFINITY || sc[j >> 1][2 * (j & 1)] != sc[j >> 1][2 * (j & 1)] ? 1.f : 0.f,
                                       sc[j >> 1][2 * (j & 1) + 1] > -INFINITY || sc[j >> 1][2 * (j & 1) + 1] != sc[j >> 1][2 * (j & 1) + 1] ? 1.f : 0.f);
                }
                const v4f hits = mfma<E>(ind, seen, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float nan = hits[i] > 0.f ? __builtin_nanf("") : 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][i] += nan;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if ((bad >> j) & 1) {
                        vs[j] = 1.f;
                        vw[j][0] = 0u;
                        if constexpr (D == 256) vw[j][1] = 0u;
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = unpack<E>(vw[j][n / 8], vs[j], (n % 8) / 2);
            v4u a0, a1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a0[j] = __builtin_amdgcn_perm(u[2 * j + 1], u[2 * j], 0x05040100u);
                a1[j] = __builtin_amdgcn_perm(u[2 * j + 1], u[2 * j], 0x07060302u);
            }
            o[n] = mfma<E>(a0, pf, o[n]);
            o[n + 1] = mfma<E>(a1, pf, o[n + 1]);
        }
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (!live) return;
    // lane: row col, dimensions (4 quarter + i) * NT + n
    const int64_t at = row * p.q_heads + hq;
    if (p.splits > 1) {
        const int64_t part = at * p.splits + split;
        if (quarter == 0) {
            p.part_ml[2 * part] = m;
            p.part_ml[2 * part + 1] = sum;
        }
        if (sum == 0.f) return;
        float* po = p.part_o + part * D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NT; n += 4)
                *reinterpret_cast<v4f*>(po + (4 * quarter + i) * NT + n) = v4f{o[n][i], o[n + 1][i], o[n + 2][i], o[n + 3][i]};
        return;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;   // NaN stays
    if (p.lse && quarter == 0) p.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at * D);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < NT; n += 2)
            out[((4 * quarter + i) * NT + n) / 2] = pack2<E>(o[n][i] * inv, o[n + 1][i] * inv);
}

// One wave per served query row and head: its splits joined in order.
template <class E, int D>
__global__ __launch_bounds__(256) void combine_kernel(AttnParams p, int64_t rows) {
    const int lane = threadIdx.x & 63;
    const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (job >= rows) return;
    const int hq = (int)(job % p.q_heads);
    const int b = (int)(job / p.q_heads / p.max_q), i = (int)(job / p.q_heads % p.max_q);
    const Rows r = rows_of(p, b);
    if (i >= r.shown) return;
    const int64_t at = (r.q0 + i) * p.q_heads + hq;
    const float* ml = p.part_ml + 2 * at * p.splits;
    float m = -INFINITY;
    for (int s = lane; s < p.splits; s += 64) m = fmaxf(m, ml[2 * s + 1] == 0.f ? -INFINITY : ml[2 * s]);
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float base = m == -INFINITY ? 0.f : m;
    float acc[D / 64] = {}, sum = 0.f;
    for (int s = 0; s < p.splits; ++s) {
        const float part = ml[2 * s + 1];
        if (part == 0.f) continue;
        const float w = exp2f(ml[2 * s] - base);
        sum += w * part;
        const float* po = p.part_o + (at * p.splits + s) * D + lane * (D / 64);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) acc[i] += w * po[i];
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (p.lse && lane == 0) p.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
    E* out = static_cast<E*>(p.out) + at * D + lane * (D / 64);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) out[i] = (E)(acc[i] * inv);
}

template <class E, int D>
gvr_status launch(const AttnParams& p, void* stream) {
    const dim3 grid((unsigned)((p.jobs + kWaves - 1) / kWaves)), block(kWaves * 64);
    if (p.selection)
        hipLaunchKernelGGL((few_rows_kernel<E, D, true>), grid, block, 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL((few_rows_kernel<E, D, false>), grid, block, 0, (hipStream_t)stream, p);
    if (hipGetLastError() != hipSuccess) return GVR_ERR_HIP;
    if (p.splits > 1) {
        const int64_t rows = (int64_t)p.sequences * p.max_q * p.q_heads;
        hipLaunchKernelGGL((combine_kernel<E, D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, (hipStream_t)stream, p,
                           rows);
        if (hipGetLastError() != hipSuccess) return GVR_ERR_HIP;
    }
    return GVR_OK;
}
template <class E>
gvr_status launch_d(const AttnParams& p, int D, void* stream) {
    return D == 64 ? launch<E, 64>(p, stream) : D == 128 ? launch<E, 128>(p, stream) : launch<E, 256>(p, stream);
}

}  // namespace

extern "C" {

gvr_status gvr_kv4_attention_workspace(const gvr_kv4_cache* cache, const gvr_kv4_attention_args* args, size_t* bytes) {
    if (!args || !bytes) return GVR_ERR_INVALID_ARG;
    *bytes = 0;
    gvr_status st = gvr_kv4::check_cache(cache, false);
    if (st != GVR_OK) return st;
    st = gvr_kv4::check_attention(*cache, *args);
    if (st != GVR_OK) return st;
    if (args->T > 0 && args->sequences > 0) *bytes = gvr_kv4::plan_attention(*cache, *args, SIZE_MAX).ws_bytes;
    return GVR_OK;
}

gvr_status gvr_kv4_attention(const gvr_kv4_cache* cache, const gvr_kv4_attention_args* args, void* workspace,
                             size_t ws_bytes, void* stream) {
    if (!args) return GVR_ERR_INVALID_ARG;
    gvr_status st = gvr_kv4::check_cache(cache, args->T > 0);
    if (st != GVR_OK) return st;
    const gvr_kv4_attention_args& a = *args;
    st = gvr_kv4::check_attention(*cache, a);
    if (st != GVR_OK) return st;
    if ((!workspace && ws_bytes > 0) || ((uintptr_t)workspace & 15)) return GVR_ERR_INVALID_ARG;
    if (a.T == 0 || a.sequences == 0) return GVR_OK;
    if (!a.q || !a.out || !a.ctx_len || (!a.block_table && a.table_width > 0)) return GVR_ERR_INVALID_ARG;
    if (((uintptr_t)a.q | (uintptr_t)a.out) & 15) return GVR_ERR_INVALID_ARG;
    const gvr_kv4::AttnPlan plan = gvr_kv4::plan_attention(*cache, a, ws_bytes);
    if (plan.jobs > gvr_kv4::kMaxCount || a.T * a.q_heads > gvr_kv4::kMaxCount) return GVR_ERR_TOO_LONG;
    AttnParams p;
    p.cache = cache->data;
    p.q = a.q, p.qt = a.q_token_stride, p.qh = a.q_head_stride;
    p.out = a.out, p.lse = a.lse;
    p.block_table = a.block_table, p.ctx_len = a.ctx_len, p.q_start = a.q_start, p.selection = a.selection;
    p.table_width = a.table_width, p.pages = cache->pages, p.T = a.T;
    p.record = gvr_kv4::record_bytes(cache->kv_heads, cache->head_dim);
    p.page_shift = gvr_kv4::log2_of(cache->page_size);
    p.kv_heads = cache->kv_heads, p.q_heads = a.q_heads, p.group = a.q_heads / cache->kv_heads;
    p.sequences = a.sequences;
    p.uniform_q = a.q_start ? 0 : (int32_t)(a.T / a.sequences);
    p.max_q = plan.max_q, p.tiles = plan.tiles, p.jobs = plan.jobs, p.splits = plan.splits, p.chunk = plan.chunk;
    p.K = a.K, p.causal = a.causal;
    p.scale2 = a.scale * kLog2e;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + (int64_t)a.T * a.q_heads * p.splits * cache->head_dim;
    return a.dtype == GVR_BF16 ? launch_d<__bf16>(p, cache->head_dim, stream)
                               : launch_d<_Float16>(p, cache->head_dim, stream);
}

}  // extern "C"
