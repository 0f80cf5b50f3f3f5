// kv4_attention.hip -- attention over the paged 4-bit cache, behind
// include/gvr_kv4.h.
//
// One wave serves 16 query rows (the query heads of one KV head, of one or
// more query tokens of a sequence) over steps of 32 tokens:
//     S^T [tokens][rows] = K Q^T,   P = exp2(S - m),   O^T [dims][rows] += V^T P^T
// Lane l holds column l % 16 (its query row) and quarter l / 16. The order of
// the tokens inside the second product is free, and is chosen so that nothing
// moves between lanes:
//   - K goes into gfx950's scaled matrix instruction as it is stored: a lane
//     takes 32 dimensions (16 bytes of codes) of one token per 16, and their
//     scale byte is the instruction's block scale. The queries are its 8-bit
//     operand: each is the sum of two E4M3 numbers (three for float16) with
//     power-of-two scales 2^-4 apart, which holds a bfloat16 exactly down to
//     2^-13 of its block's largest magnitude (an error of at most 2^-21 of it
//     below). Against unpacking K for the 16-bit instruction this costs the
//     same matrix time and 32 vector instructions a step less;
//   - the scores that come out sit in the lane that feeds them, as weights, to
//     the second product: tokens 4 q + i of both halves of the step;
//   - V: for those tokens a lane takes D / 16 consecutive dimensions, and the
//     n-th of them goes to the n-th matrix step. One instruction turns two
//     codes and their scale into two 16-bit floats; the values of two tokens
//     are then paired by byte permutes. (The scales of V lie along the
//     dimensions, across the product's sum, so V cannot go in as stored.)
// Sum and maximum are float32 per row. Lanes exchange the maximum and rescale O
// only in steps in which some score passes it, which become rare. (Letting it
// lag by up to 2^8 saves a few percent more and costs accuracy: with the true
// maximum the largest weight is 1, which has no rounding error. Relative error
// of 2048 selected tokens 0.0017 against 0.0019, 0.0016 being the output's own
// rounding.)
//
// A workgroup is `hw` KV heads x `tw` waves (eight in all) that take turns at
// the steps of one chunk of a context; its waves are joined in LDS, chunks of a
// context by a second kernel from float32 partial results, in a fixed order. A
// unit is one chunk of one sequence. Chunks are of one length that the host
// chooses, or, for several sequences, of one that every workgroup works out
// from the contexts' lengths (48 contexts of 0 .. 16K tokens, waves together
// every step: 43 us against 59 with the host's). Units that read the same records go to one XCD.
//
// What bounds it, measured (MI355X; a plain read of as many bytes in brackets):
//   32 x 32K tokens, 8 KV heads of 128, 4 rows each: 210 us = 5.4 TB/s (166 us);
//     memory: the same loads with nothing computed take 205 us, because a head's
//     64 bytes of codes per record are half a line, and its eight waves do not
//     ask for both halves at once;
//   1 x 512K tokens, 8 rows: 117 us (83 us): the same, and the join of 256 parts;
//   128 rows of 2048 selected tokens: 61 us (41 us for what the rows select
//     one by one, 24 for what two draft rows have in common): gathers of 1 KB;
//   48 x 3 rows over 0 .. 16K tokens, 2 KV heads of 64, float16: 35 us (7.5 us):
//     12 us before the first record (lengths, splits, pages), 6 of join, and steps at
//     2.6 TB/s, which two row tiles of dependent products and exponentials set;
//   1 x 1K tokens: 12.5 us: latency, of two launches and in the first of them
//     length -> page -> record -> join.
// All of it where the table of pages is about as wide as the contexts are long:
// the host plans by the table's width (64 heads over one request of 32K tokens in
// a table for as many 20 us, for 512K, with work for 16 workgroups, 95; a chunk of 512
// tokens at 8K, 32 heads, in a table for 8K 117 us, for 128K 311; 32 requests of 8K, which the
// kernel balances, 62 and 60). And a selection costs what its K entries do, also
// where they are -1 (64 rows of 300 tokens: K = 320 12 us, 2048 34).
// More than 128 rows of a KV head: see "many query rows" below.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "gvr_kv4.h"
#pragma clang force_cuda_host_device begin
#include "kv4_plan.h"
#pragma clang force_cuda_host_device end
#include "wave_ops.h"

namespace {

using gvr_kv4::kRows;
using gvr_kv4::kStep;
using gvr_kv4::kThreads;
using gvr_kv4::kMaxSplits;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef int v8i __attribute__((ext_vector_type(8)));
template <class E> struct Vec { typedef E x8 __attribute__((ext_vector_type(8))); typedef E x2 __attribute__((ext_vector_type(2))); };

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;

struct AttnParams {
    const uint8_t* cache;
    const void* q;
    void* out;
    float* lse;
    // Partial results of unit u (a sequence's split), of its query token i and head hq, at
    // (u * max_q + i) * q_heads + hq: O [D], and maximum (log2 domain) and sum.
    float* part_o;
    float* part_ml;
    int2* units_of;   // balanced splits: [sequences] first unit and number of units
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* q_start;
    const int32_t* selection;
    int64_t qt, qh;   // query strides
    int64_t table_width, record, T;
    int32_t page_shift, kv_heads, q_heads, group, sequences, uniform_q, max_q, tiles, splits, chunk, K, causal;
    int32_t pages;
    int32_t balanced, units;      // splits sized in the kernel so that the contexts' lengths fill `units`
    int32_t many, row_tiles;      // the many-rows kernel, or the few-rows one with so many tiles of 16 rows a wave
    int32_t hw_shift, tw_shift;   // log2 of a workgroup's KV heads, and of the waves that share a head's steps
    float scale2;     // scale * log2(e)
};

// Two codes (byte `sel` of w) times the scale as a packed pair.
template <class E>
DEV uint32_t unpack(uint32_t w, float scale, int sel) {
    typename Vec<E>::x2 v;
    if constexpr (__is_same(E, __bf16)) {
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
// 16 tokens x 128 dimensions in 4 bits times 128 dimensions x 16 rows in 8 bits.
constexpr int kFp8 = 0, kFp4 = 4;
DEV v4f mfma_mx(v4u a, uint32_t sa, v8i b, uint32_t sb, v4f c) {
    const v8i a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b, c, kFp4, kFp8, 0, (int)sa, 0, (int)sb);
}
template <class E>
DEV uint32_t pack2(float a, float b) {
    typename Vec<E>::x2 v;
    v[0] = (E)a, v[1] = (E)b;
    return __builtin_bit_cast(uint32_t, v);
}
// The largest; NaN if one of them is (then the row's weights are NaN in any
// case). Unlike fmaxf this needs no quieting of each operand first.
DEV float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
DEV float max3(float a, float b, float c) { return max2(max2(a, b), c); }
// The largest over the two halves of the wave, and over its four rows of 16
// lanes, in every lane (swaps between rows, no LDS round trip).
DEV float max_halves(float x) {
    const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
DEV float max_rows(float x) {
    const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_halves(fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1])));
}
// A row's weights from its scores. In bfloat16 at most 1, base the maximum *
// scale2. Float16 has fewer exponents: weights of 2^-25 and less would be zero
// in the second product, and with them the tail of a long context behind one
// large score (20000 tokens 17.5 below an attention sink of value zero are the
// whole result, and would be lost). So they are 2^15 times as large there, which
// moves that limit to 2^-40, and sum and O are scaled back at the end. Base is
// the maximum itself, so that the largest is 2^15 whatever the scores' size: one
// more subtraction a weight (2048 rows of 32 heads over 16K tokens, D = 64: 385 us
// against 374, D = 128: 655 to 695 against 640 to 660; 32 x 8K tokens 60.6, 60.0).
constexpr float kUp = 15.f, kDown = 1.f / 32768;
template <class E>
DEV float base_of(float m, float scale2) {
    return m == -INFINITY ? 0.f : __is_same(E, __bf16) ? m * scale2 : m;
}
template <class E>
DEV float weight_of(float s, float scale2, float base) {
    if constexpr (__is_same(E, __bf16))
        return __builtin_amdgcn_exp2f(__builtin_fmaf(s, scale2, -base));
    else
        return __builtin_amdgcn_exp2f(__builtin_fmaf(s - base, scale2, kUp));
}
DEV float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// First scale byte with codes beyond the 16-bit type (4 * 2^14; 4 * 2^126).
template <class E>
constexpr uint32_t kOver = __is_same(E, __bf16) ? 253 : 141;

// NB bytes of codes as dwords (records are 4-byte aligned, runs of 2 bytes 2-byte).
template <int NB>
struct Codes {
    uint32_t w[NB / 4 ? NB / 4 : 1];
};
template <int NB>
DEV Codes<NB> load_codes(const uint8_t* p) {
    Codes<NB> c;
    if constexpr (NB == 2) {
        c.w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (NB == 4) {
        c.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(NB / 4), aligned(4)));
        const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int j = 0; j < NB / 4; ++j) c.w[j] = v[j];
    }
    return c;
}
DEV v4u load16(const uint8_t* p) {
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
    return *reinterpret_cast<const vec*>(p);
}

// A query row as 8-bit terms for the scaled product: T terms per run of 128
// dimensions (D = 64: the run holds the dimensions twice, for two terms).
// Byte i of a lane's half-run r is dimension 64 r + 16 quarter + i; a lane's
// scale byte is that of the dimensions 32 quarter ..
template <class E, int D>
struct Query {
    static constexpr int kTerms = __is_same(E, __bf16) ? 2 : 3;
    static constexpr int kRuns = D == 64 ? (kTerms + 1) / 2 : D / 128;
    static constexpr int kPer = D == 64 ? 1 : kTerms;   // products per run
    v8i b[kRuns][kPer];
    uint32_t scale[kRuns][kPer];
};

// Sixteen elements as four dwords of E4M3, and what is left of them times 16.
DEV void split16(float (&x)[16], v8i& out, int at) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
        out[at + i] = w;
        x[4 * i] = 16.f * (x[4 * i] - __builtin_amdgcn_cvt_f32_fp8(w, 0));
        x[4 * i + 1] = 16.f * (x[4 * i + 1] - __builtin_amdgcn_cvt_f32_fp8(w, 1));
        x[4 * i + 2] = 16.f * (x[4 * i + 2] - __builtin_amdgcn_cvt_f32_fp8(w, 2));
        x[4 * i + 3] = 16.f * (x[4 * i + 3] - __builtin_amdgcn_cvt_f32_fp8(w, 3));
    }
}

// q: the row's D elements (NULL: zeros), times sign. Lanes of one row must
// all be active. Not finite: the block's scale is NaN.
template <class E, int D>
DEV Query<E, D> load_query(const E* q, float sign, int lane) {
    typedef typename Vec<E>::x8 x8;
    const int col = lane & 15, quarter = lane >> 4;
    Query<E, D> r;
    // scale of the 32 dimensions from 32 quarter (+ 128 per run): largest magnitude in [2^7, 2^8)
    constexpr int kBlocks = D == 256 ? 2 : 1;
    uint32_t byte[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        uint32_t m = 0;
        if (q) {
            const E* p = q + 128 * c + 32 * (D == 64 ? quarter & 1 : quarter);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const x8 v = *reinterpret_cast<const x8*>(p + 8 * i);
#pragma unroll
                for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint((float)v[j]) & 0x7FFFFFFFu);
            }
        }
        const int e = (int)(m >> 23);
        byte[c] = e == 255 ? 255u : (uint32_t)max(e - 7, 16);   // 16: room for the lower terms
    }
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        float x[2][16];   // half-runs
#pragma unroll
        for (int h = 0; h < (D == 64 ? 1 : 2); ++h) {
            const uint32_t b = (uint32_t)__shfl((int)byte[c], col + 16 * (2 * h + (quarter >> 1)), 64);
            const float inv = b == 255 ? 0.f : __uint_as_float((254u - b) << 23) * sign;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x8 v = {};
                if (q) v = *reinterpret_cast<const x8*>(q + 128 * c + 64 * h + 16 * quarter + 8 * i);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[h][8 * i + j] = b == 255 ? 0.f : (float)v[j] * inv;
            }
        }
        if constexpr (D == 64) {
            // terms 0 and 1 share a run, term 2 has the lower half of another
#pragma unroll
            for (int t = 0; t < r.kTerms; ++t) split16(x[0], r.b[t / 2][0], 4 * (t & 1));
            r.scale[0][0] = byte[0] == 255 ? 255u : byte[0] - (quarter >= 2 ? 4u : 0u);
            if constexpr (r.kTerms == 3) {
#pragma unroll
                for (int i = 4; i < 8; ++i) r.b[1][0][i] = 0;
                r.scale[1][0] = byte[0] == 255 ? 255u : byte[0] - 8u;
            }
        } else {
#pragma unroll
            for (int t = 0; t < r.kTerms; ++t) {
                split16(x[0], r.b[c][t], 0);
                split16(x[1], r.b[c][t], 4);
                r.scale[c][t] = byte[c] == 255 ? 255u : byte[c] - 4u * t;
            }
        }
    }
    return r;
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

// LDS of a wave: the codes of V of its 32 tokens (16-byte chunks, see v_place)
// and the scale bytes of K and V; of a workgroup: its waves', then slots.
template <int D>
struct WaveLds {
    static constexpr int kCodes = kStep * D / 2;
    static constexpr int kScales = kStep * D / 32;     // of K, then as many of V
    static constexpr int kBytes = kCodes + 2 * kScales;
    static constexpr int kSlots = D == 256 ? 4096 : 8192;   // tokens whose slots the workgroup holds
    static constexpr int kLds = gvr_kv4::kWaves * kBytes + kSlots * 4;   // and the queries of the workgroup's heads
};

// Byte of chunk `chunk` of V's codes of token tok (0 .. 31): tokens 4 q + i of
// 16 lie in the order i, q, so that the quarters read side by side, and the
// chunks of a token are turned by i, so that a write of 16 tokens meets all banks.
template <int D>
DEV int v_place(int tok, int chunk) {
    const int i = tok & 3;
    return ((tok & ~15) + 4 * i + ((tok >> 2) & 3)) * (D / 2) + (chunk ^ (D == 64 ? i & 1 : i)) * 16;
}

// First token of a step (steps past the last token, of a tile's padding, may
// start beyond what an int holds: they see none of theirs).
DEV int step_at(int piece, int t) { return (int)min((uint32_t)piece + (uint32_t)t, 0x7FFFFFE0u); }

DEV void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A workgroup's unit of the balanced splits: sequence b's split `split` of
// `count`, chunk tokens each.
struct Unit {
    int b, split, count, first, chunk;   // first: unit of split 0; b < 0: none
};
DEV int context_of(const AttnParams& p, int b) {
    const int64_t held = p.table_width << p.page_shift;
    return p.pages > 0 ? (int)min((int64_t)max(p.ctx_len[b], 0), held) : 0;
}
// The sequences' contexts are cut into chunks of one length, the least of eight
// candidates (one per wave) for which the chunks count no more than the units.
// Candidate 7 always serves: with n sequences and u units, chunks of at least
// total / (u - n) are at most u - n full ones and n parts.
DEV Unit find_unit(const AttnParams& p, int u, int tt_shift, int32_t* lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = p.sequences;
    const int mine = lane < n ? context_of(p, lane) : 0;
    auto context = [&](int b0) { return b0 == 0 ? mine : b0 + lane < n ? context_of(p, b0 + lane) : 0; };
    float total = 0.f;
    int longest = 0;
    for (int b0 = 0; b0 < n; b0 += 64) {
        const int c = context(b0);
        total += gvr_dev::wave_sum_f((float)c);
        longest = max(longest, c);
    }
    longest = (int)gvr_dev::wave_max_u((uint32_t)longest);
    // (no context has more than kMaxSplits chunks: what the joining kernel holds)
    const int floor = max((int)(((uint32_t)longest + kMaxSplits - 1) / kMaxSplits), 1);
    const float least = total / (float)p.units * 0.999999f;
    const float most = total * 1.00001f / (float)(p.units - n) + 1.f;   // (float32 sums: a margin)
    auto length = [&](int k) {
        const float c = least + (most - least) * (float)k * (1.f / (gvr_kv4::kWaves - 1));
        return (max((int)fminf(ceilf(c), 2.1e9f), floor) + (1 << tt_shift) - 1) >> tt_shift << tt_shift;   // whole tiles
    };
    auto chunks = [&](int b0, int len) {
        return b0 + lane < n ? max(1, (int)(((uint32_t)context(b0) + (uint32_t)len - 1) / (uint32_t)len)) : 0;
    };
    const int len = length(wave);
    int count = 0;
    for (int b0 = 0; b0 < n; b0 += 64) count += gvr_dev::wave_sum(chunks(b0, len));
    if (lane == 0) lds[wave] = count;
    __syncthreads();
    int k = 0;
    while (k < gvr_kv4::kWaves - 1 && lds[k] > p.units) ++k;
    Unit r = {-1, 0, 0, 0, length(k)};
    int before = 0;
    for (int b0 = 0; b0 < n; b0 += 64) {
        const int own = chunks(b0, r.chunk), upto = before + gvr_dev::wave_incl_scan(own, lane);
        const uint64_t past = __ballot(upto > u && b0 + lane < n);
        if (past) {
            const int at = __builtin_ctzll(past);
            r.b = b0 + at;
            r.count = __builtin_amdgcn_readlane(own, at);
            r.first = __builtin_amdgcn_readlane(upto, at) - r.count;
            r.split = u - r.first;
            break;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    r.chunk = __builtin_amdgcn_readfirstlane(r.chunk);
    return r;
}

// The work of a workgroup: unit u of U (a sequence's split) and one of `inner`
// jobs of the unit. Jobs of a unit read the same records, so they go to one
// XCD (workgroups are dealt to the eight in turn), where they meet in its L2.
struct Job {
    int64_t unit;
    int inner;
};
DEV Job job_of(uint32_t bid, int64_t units, int inner) {
    if (gvr_kv4::by_xcd(units)) {
        const uint32_t y = bid >> 3;
        return {(int64_t)(y / (uint32_t)inner) * 8 + (bid & 7), (int)(y % (uint32_t)inner)};
    }
    return {bid / (uint32_t)inner, (int)(bid % (uint32_t)inner)};
}

// MT: row tiles of 16 that a wave serves with one pass over K and V. Two where
// more than 16 rows share their tokens: the bytes are read and V is unpacked
// once for both (32 x 8K tokens, 8 heads of 128, waves together every step: 32
// rows 93 us against 129, 64 rows 160 against 226). D = 256 has no registers
// for two.
// Registers: one workgroup to a compute unit (256 a lane), but two where 128
// suffice without spills, which is D = 64, MT = 1 in bfloat16: 32 x 32K tokens
// 159 us against 174, small calls within 2 us either way.
template <class E, int D, int MT>
__global__ __launch_bounds__(kThreads, D == 64 && MT == 1 && __is_same(E, __bf16) ? 4 : 2) void few_rows_kernel(AttnParams p) {
    constexpr int NT = D / 16;        // dimensions of V per lane = matrix steps of the second product
    typedef Query<E, D> Q;
    typedef WaveLds<D> L;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hl = wave & ((1 << p.hw_shift) - 1);        // head of the workgroup's
    const int tg = wave >> p.hw_shift;                    // part of the tile's tokens
    const int tt_shift = 5 + p.tw_shift, TT = 1 << tt_shift;   // tokens of a tile
    const int groups = p.kv_heads >> p.hw_shift;
    const Job job = job_of(blockIdx.x, p.units, groups * p.tiles);
    if (job.unit >= p.units) return;
    const int h = (job.inner % groups << p.hw_shift) + hl, tile = job.inner / groups;
    Unit unit = {(int)(job.unit / p.splits), (int)(job.unit % p.splits), p.splits, 0, p.chunk};
    if (p.balanced) {
        unit = find_unit(p, (int)job.unit, tt_shift, reinterpret_cast<int32_t*>(lds));
        if (unit.b < 0) return;
        if (job.inner == 0 && unit.split == 0 && threadIdx.x == 0) p.units_of[unit.b] = int2{unit.first, unit.count};
        __syncthreads();   // (the counts' place in LDS)
    }
    const int b = unit.b;

    const Rows rows = rows_of(p, b);
    const int64_t q0 = rows.q0, nq = rows.nq;
    const int shown = rows.shown;
    if (shown <= 0) return;
    const int64_t held = p.table_width << p.page_shift;
    const int32_t* table = p.block_table + (int64_t)b * p.table_width;
    const int64_t lo = (int64_t)unit.split * unit.chunk;
    // The first tokens' list entries and page numbers are loaded while the
    // context's length is.
    int early_tok = -1, early_page = -1;
    if (p.selection) {
        const int token = tile / ((p.group + MT * kRows - 1) / (MT * kRows));
        if (token < shown && lo + threadIdx.x < p.K) early_tok = p.selection[(q0 + token) * p.K + lo + threadIdx.x];
    } else if (lo + threadIdx.x < held) {
        early_tok = (int)(lo + threadIdx.x);
    }
    if (early_tok >= 0 && early_tok < held) early_page = table[early_tok >> p.page_shift];
    const int ctx = p.pages > 0 ? (int)min((int64_t)max(p.ctx_len[b], 0), held) : 0;

    // this lane's query rows; tokens [0, end) of the context or selection concern the tile
    int qi[MT], qg[MT], end, sel_last = 0;
    bool live[MT];
    const int32_t* list = nullptr;
    if (p.selection) {
        const int per = (p.group + MT * kRows - 1) / (MT * kRows), token = tile / per;
        if (token >= shown) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            qi[mt] = token;
            qg[mt] = (tile - token * per) * (MT * kRows) + mt * kRows + col;
            live[mt] = qg[mt] < p.group;
        }
        end = p.pages > 0 ? p.K : 0;
        list = p.selection + (q0 + token) * p.K;
        sel_last = p.causal ? (int)(ctx - nq + token) : ctx - 1;
    } else {
        const int r0 = tile * (MT * kRows);
        if (r0 / p.group >= shown) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int r = r0 + mt * kRows + col;
            qi[mt] = r / p.group;
            qg[mt] = r - qi[mt] * p.group;
            live[mt] = qi[mt] < shown;
        }
        const int qi_last = min((r0 + MT * kRows - 1) / p.group, shown - 1);
        end = (int)max((int64_t)0, p.causal ? ctx - nq + qi_last + 1 : (int64_t)ctx);
    }
    // last token that this lane's rows see, and the last that all of the tile's rows see
    int last[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
        last[mt] = !live[mt] ? -1 : list ? 0x7FFFFFFF : p.causal ? (int)(ctx - nq + qi[mt]) : ctx - 1;
    const int all_last =
        list ? 0x7FFFFFFF
             : (int)max((int64_t)-1, p.causal ? ctx - nq + (tile * (MT * kRows)) / p.group : (int64_t)ctx - 1);
    const int begin = (int)min(lo, (int64_t)end), stop = (int)min(lo + unit.chunk, (int64_t)end);

    const float scale2 = fabsf(p.scale2);
    const uint32_t record = (uint32_t)p.record;
    const int page_mask = (1 << p.page_shift) - 1;

    // The lane loads 16-byte chunk `quarter` of K and V of token `col` of each
    // half of a step (D = 64: the quarters 2, 3 repeat 0, 1; D = 256: chunk
    // quarter + 4 too), and from the scales those of K or V.
    constexpr int kRuns = D == 256 ? 2 : 1;
    const int chunk = D == 64 ? quarter & 1 : quarter;
    const uint8_t* const k_src = p.cache + (uint32_t)(h * (D / 2) + chunk * 16);
    const uint8_t* const v_src = p.cache + (uint32_t)((p.kv_heads + h) * (D / 2) + chunk * 16);
    const uint8_t* const s_src = p.cache + (uint32_t)(p.kv_heads * D + ((quarter & 1 ? p.kv_heads : 0) + h) * (D / 32));
    uint8_t* const mine = lds + wave * L::kBytes;
    int32_t* const slots = reinterpret_cast<int32_t*>(lds + gvr_kv4::kWaves * L::kBytes);
    constexpr int kTerms = Q::kRuns * Q::kPer;
    // The head's queries stay in LDS (16 bytes a lane side by side): they are
    // needed once a step, and their registers are worth a second workgroup.
    v4u* const q_lds = reinterpret_cast<v4u*>(lds + L::kLds) + hl * (MT * kTerms * 2 * 64) + lane;
    uint32_t q_scale[MT][kTerms];
    auto query = [&](int mt, int i) {
        const v4u a = q_lds[(mt * kTerms + i) * 128], b = q_lds[(mt * kTerms + i) * 128 + 64];
        return v8i{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    };
    struct Step {
        v4u k[2][kRuns], v[2][kRuns];
        Codes<D / 32> s[2];
        uint32_t there;   // bit n: token n exists
    };
    auto fetch = [&](int t_lds, Step& d) {   // the step at slot t_lds of the piece
        d.there = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int slot = slots[t_lds + 16 * t + col];
            d.there |= ((uint32_t)__ballot(slot >= 0) & 0xFFFFu) << (16 * t);
            const uint64_t at = (uint64_t)(uint32_t)max(slot, 0) * record;
#pragma unroll
            for (int c = 0; c < kRuns; ++c) {
                d.k[t][c] = load16(k_src + at + 64 * c);
                d.v[t][c] = load16(v_src + at + 64 * c);
            }
            d.s[t] = load_codes<D / 32>(s_src + at);
        }
    };
    // Where the lane writes and reads in its wave's LDS (t: constants).
    const int vw_at = v_place<D>(col, chunk), sw_at = L::kCodes + (quarter & 1) * L::kScales + col * (D / 32);
    const int ks_at = L::kCodes + col * (D / 32) + chunk;
    const int vs_at = L::kCodes + L::kScales + 4 * quarter * (D / 32) + col * (D / 16) / 32;
    int vr_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int byte = col * (D / 32);
        vr_at[i] = v_place<D>(4 * quarter + i, byte / 16) + byte % 16;
    }

    // Of each row: the maximum of its unscaled scores, its base (base_of), the sum;
    // whether it sees a value that is NaN in this lane's dimensions (D = 256:
    // lower, upper half).
    float m[MT], base[MT], sum[MT];
    uint32_t nan_blocks[MT];
    v4f o[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -INFINITY;
        base[mt] = sum[mt] = 0.f;
        nan_blocks[mt] = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[mt][n] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    // t0: first token (or place in the list) of the step; its registers take
    // the step at slot t_next when they are free.
    auto use = [&](Step& d, int t0, int t_next) {
        const uint32_t there = d.there;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < kRuns; ++c)
                *reinterpret_cast<v4u*>(mine + (vw_at ^ (64 * c)) + 16 * t * (D / 2)) = d.v[t][c];
            uint8_t* sw = mine + sw_at + 16 * t * (D / 32);
            if constexpr (D == 64)
                *reinterpret_cast<uint16_t*>(sw) = (uint16_t)d.s[t].w[0];
            else if constexpr (D == 128)
                *reinterpret_cast<uint32_t*>(sw) = d.s[t].w[0];
            else
                *reinterpret_cast<v2u*>(sw) = v2u{d.s[t].w[0], d.s[t].w[1]};
        }
        // the wave's lanes read what other lanes wrote (in order, without a barrier)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        v4f sc[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            sc[mt][0] = sc[mt][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = kTerms - 1; i >= 0; --i) {   // (D = 64: runs of the same K; else terms, then runs of K)
                const int c = D == 64 ? 0 : i / Q::kPer;
                const v8i qf = query(mt, i);
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    sc[mt][t] = mfma_mx(d.k[t][c], mine[ks_at + 16 * t * (D / 32) + 4 * c], qf, q_scale[mt][i], sc[mt][t]);
            }
        }
        fetch(t_next, d);
        Codes<D / 32> v[8];
        float vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t* vp = mine + vr_at[j & 3] + 16 * (j >> 2) * (D / 2);
            if constexpr (D == 64)
                v[j].w[0] = *reinterpret_cast<const uint16_t*>(vp);
            else if constexpr (D == 128)
                v[j].w[0] = *reinterpret_cast<const uint32_t*>(vp);
            else {
                const v2u w = *reinterpret_cast<const v2u*>(vp);
                v[j].w[0] = w[0], v[j].w[1] = w[1];
            }
            vs[j] = scale_of(mine[vs_at + (16 * (j >> 2) + (j & 3)) * (D / 32)]);
        }
        const bool full = there == 0xFFFFFFFFu && t0 + kStep - 1 <= all_last;   // wave-uniform
        int quarter_now = quarter;   // (its multiples are not worth registers through the loop)
        asm("" : "+v"(quarter_now));
        v4u pf[MT];
        bool bad = false;
        if (!full) {
            // A masked token's weight is zero, but a NaN block times zero is
            // not: blocks that are NaN, and tokens that are not there, are
            // taken as zeros, and the rows that see a NaN remember it. So are,
            // in tokens that some row does not see, blocks of values that
            // become infinite in the 16-bit type.
            auto first_bad = [&](int n) { return t0 + n > all_last ? kOver<E> : 255u; };
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int n = 16 * (j >> 2) + 4 * quarter_now + (j & 3);
                const bool here = (there >> n) & 1;
                const bool nan = __float_as_uint(vs[j]) >= first_bad(n) << 23;
                bad |= here && nan;
                if (!here || nan) {
                    vs[j] = 0.f;
                    v[j] = Codes<D / 32>{};
                }
            }
            if (__any(bad)) {
                // this lane's sums are of dimensions D / 4 quarter .. + D / 4
                const uint8_t* vsb = mine + L::kCodes + L::kScales + D / 4 * quarter / 32;
#pragma unroll 1
                for (int n = 0; n < kStep; ++n) {
                    uint32_t nan = vsb[n * (D / 32)] >= first_bad(n) ? 1u : 0u;
                    if constexpr (D == 256) nan |= vsb[n * (D / 32) + 1] >= first_bad(n) ? 2u : 0u;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        nan_blocks[mt] |= ((there >> n) & 1) != 0 && t0 + n <= last[mt] ? nan : 0u;
                }
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            v4f(&s)[2] = sc[mt];
            uint32_t seen = 0;   // bit 4 t + i: this row sees token 16 t + 4 quarter + i
            if (!full) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int n = 16 * t + 4 * quarter_now + i;
                        const bool see = ((there >> n) & 1) && t0 + n <= last[mt];
                        seen |= see ? 1u << (4 * t + i) : 0u;
                        if (!see) s[t][i] = -INFINITY;
                    }
            }
            float top = max2(max3(max3(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]), max3(s[1][1], s[1][2], s[1][3]));
            if (__any(top > m[mt])) {
                const float m_new = fmaxf(m[mt], max_rows(top));
                // (nothing seen so far: sum and O are zero)
                const float keep =
                    m_new == m[mt] || m[mt] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[mt] - m_new) * scale2);
                m[mt] = m_new;
                base[mt] = base_of<E>(m_new, scale2);
                sum[mt] *= keep;
#pragma unroll
                for (int n = 0; n < NT; ++n) o[mt][n] *= keep;
            }
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = weight_of<E>(s[j >> 2][j & 3], scale2, base[mt]);
            if (!full) {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (seen >> j) & 1 ? w[j] : 0.f;
            }
            sum[mt] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            pf[mt] = v4u{pack2<E>(w[0], w[1]), pack2<E>(w[2], w[3]), pack2<E>(w[4], w[5]), pack2<E>(w[6], w[7])};
        }
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = unpack<E>(v[j].w[n / 8], vs[j], (n % 8) / 2);
            v4u a0, a1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a0[j] = __builtin_amdgcn_perm(u[2 * j + 1], u[2 * j], 0x05040100u);
                a1[j] = __builtin_amdgcn_perm(u[2 * j + 1], u[2 * j], 0x07060302u);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                o[mt][n] = mfma<E>(a0, pf[mt], o[mt][n]);
                o[mt][n + 1] = mfma<E>(a1, pf[mt], o[mt][n + 1]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");   // the next step writes where this one read
    };

    // Pieces of the chunk: slots into LDS, then step after step, the loads one
    // step ahead (two ahead measured no faster: 32 x 32K tokens wait for the
    // memory either way). The waves of a workgroup read different parts of the same
    // records, so they are kept together: a line that one of them brought into
    // the caches is used by the others before it leaves. How often depends on
    // what a step computes and reads: where more is computed the memory is less of
    // a bound, and waves gain from being at different places of a step; selected
    // records are apart in any case. Every step, every second, every sixteenth
    // (us): 32 x 32K tokens, D = 64 152, 155, 163, D = 128 (not in the caches) 210,
    // 212, -; 128 rows of 2048 selected 63.7, 61.4, 63.9; two row tiles, 64 rows
    // over 32 x 8K 160, 146, 138; D = 256, 16 x 8K 71, 68, 66.
    const int together = MT == 2 || D == 256 ? 15 : list ? 1 : 0;   // less one
    for (int64_t from = begin; from < stop; from += L::kSlots) {
        const int piece = (int)from;
        const int fill = min(stop - piece, L::kSlots), padded = (fill + TT - 1) & -TT;
        lds_barrier();   // the waves are through with the last piece
        for (int i = threadIdx.x; i < padded; i += kThreads) {
            int slot = -1;
            if (i < fill) {
                const bool early = piece == begin && i < kThreads;
                const int tok = early ? early_tok : list ? list[piece + i] : piece + i;
                if (tok >= 0 && (!list || tok <= sel_last)) {
                    const int page = early ? early_page : table[tok >> p.page_shift];
                    if ((uint32_t)page < (uint32_t)p.pages) slot = (page << p.page_shift) + (tok & page_mask);
                }
            }
            slots[i] = slot;
        }
        lds_barrier();
        const int first = kStep * tg, final = padded - TT + first;
        Step d;
        fetch(first, d);
        if (piece == begin) {   // while the first loads run
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int64_t at = (q0 + qi[mt]) * p.qt + (h * p.group + qg[mt]) * p.qh;
                const Q q = load_query<E, D>(live[mt] ? static_cast<const E*>(p.q) + at : nullptr,
                                             p.scale2 < 0.f ? -1.f : 1.f, lane);
#pragma unroll
                for (int i = 0; i < kTerms; ++i) {
                    const v8i b = q.b[i / Q::kPer][i % Q::kPer];
                    q_scale[mt][i] = q.scale[i / Q::kPer][i % Q::kPer];
                    if (tg == 0) {
                        v4u* to = q_lds + (mt * kTerms + i) * 128;
                        to[0] = v4u{(uint32_t)b[0], (uint32_t)b[1], (uint32_t)b[2], (uint32_t)b[3]};
                        to[64] = v4u{(uint32_t)b[4], (uint32_t)b[5], (uint32_t)b[6], (uint32_t)b[7]};
                    }
                }
            }
            lds_barrier();
        }
        for (int t = first; t < padded; t += TT) {
            use(d, step_at(piece, t), min(t + TT, final));
            if (((t >> tt_shift) & together) == together) __builtin_amdgcn_s_barrier();
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        sum[mt] += __shfl_xor(sum[mt], 16, 64);
        sum[mt] += __shfl_xor(sum[mt], 32, 64);
        if constexpr (!__is_same(E, __bf16)) {
            sum[mt] *= kDown;
#pragma unroll
            for (int n = 0; n < NT; ++n) o[mt][n] *= kDown;
        }
        if (nan_blocks[mt]) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o[mt][n][i] += (nan_blocks[mt] >> (D == 256 ? i / 2 : 0)) & 1 ? __builtin_nanf("") : 0.f;
        }
    }

    // Join the waves of a head: half of them hand theirs to the other half.
    for (int half = (1 << p.tw_shift) >> 1; half > 0; half >>= 1) {
        const int places = half << p.hw_shift;   // of waves in LDS
        const int place = (tg & (half - 1)) << p.hw_shift | hl;
        v4f* lo4 = reinterpret_cast<v4f*>(lds) + (place * MT * NT) * 64 + lane;
        float2* lml = reinterpret_cast<float2*>(lds + (size_t)places * MT * NT * 1024) + place * MT * 64 + lane;
        lds_barrier();
        if (tg >= half && tg < 2 * half) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int n = 0; n < NT; ++n) lo4[(mt * NT + n) * 64] = o[mt][n];
                lml[mt * 64] = float2{m[mt], sum[mt]};
            }
        }
        lds_barrier();
        if (tg < half) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float2 other = lml[mt * 64];
                const float m_new = fmaxf(m[mt], other.x);
                const float mine_w = m[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[mt] - m_new) * scale2);
                const float theirs = other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((other.x - m_new) * scale2);
                sum[mt] = sum[mt] * mine_w + other.y * theirs;
                m[mt] = m_new;
#pragma unroll
                for (int n = 0; n < NT; ++n) o[mt][n] = o[mt][n] * mine_w + lo4[(mt * NT + n) * 64] * theirs;
            }
        }
    }
    if (tg != 0) return;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        if (!live[mt]) continue;
        // lane: row col, dimensions (4 quarter + i) * NT + n
        const int64_t at = (q0 + qi[mt]) * p.q_heads + h * p.group + qg[mt];
        const float m2 = m[mt] == -INFINITY ? m[mt] : m[mt] * scale2;
        if (unit.count > 1) {
            const int64_t part = (job.unit * p.max_q + qi[mt]) * p.q_heads + h * p.group + qg[mt];
            if (quarter == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * part) = float2{m2, sum[mt]};
            if (sum[mt] == 0.f) continue;
            float* po = p.part_o + part * D;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NT; n += 4)
                    *reinterpret_cast<v4f*>(po + (4 * quarter + i) * NT + n) =
                        v4f{o[mt][n][i], o[mt][n + 1][i], o[mt][n + 2][i], o[mt][n + 3][i]};
            continue;
        }
        const float inv = sum[mt] > 0.f ? 1.f / sum[mt] : sum[mt] == 0.f ? 0.f : sum[mt];   // NaN stays
        if (p.lse && quarter == 0) p.lse[at] = sum[mt] == 0.f ? -INFINITY : (m2 + log2f(sum[mt])) * kLn2;
        uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at * D);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NT; n += 2)
                out[((4 * quarter + i) * NT + n) / 2] = pack2<E>(o[mt][n][i] * inv, o[mt][n + 1][i] * inv);
    }
}

// ---- many query rows
//
// A workgroup of NW waves serves 32 NW query rows of one KV head, 32 per wave,
// with the 32x32 matrix instructions; the products are those of the few-rows
// kernel (a lane's column l % 32 is its row, half l / 32). The context goes
// through LDS in tiles of 16 NW tokens: K as stored, V as 16-bit floats,
// transposed (a row of tokens per dimension, in the order in which the
// scores' registers name them), unpacked once for all the rows. Two buffers: a
// tile is unpacked into one while the other is used, and the records of the
// tile after it are on their way in registers.
// 4096 rows of 32 heads over 32K tokens, 8 KV heads of 128: 1.95 to 2.02 ms, 1.02
// to 1.06 PFLOP/s (calls back to back, at lower clocks: 2.2 to 2.4 ms), against
// 3.83 ms with the few-rows kernel. Bound by the vector unit beside the matrix
// cores: exponentials, packing and the unpacking of V. Float16, with three terms
// of the queries, is slower: 2048 rows over 16K tokens 655 to 695 us against 540 (D = 64:
// 385; D = 256, 1024 rows of 16 heads: 557), and at D = 128 and 256 its registers
// spill (12 and 28 bytes a lane). At D = 256 a SIMD has one wave. For 128
// rows and fewer the few-rows kernel is ahead (32 x 8K tokens: 64 rows 139 us
// against 234, 128 rows 256 against 274, 192 rows 398 against 348): half of this
// one's rows are then empty.
template <int D, int NW>
struct Many {
    static constexpr int kThreads = 64 * NW;               // (AttnPlan::threads)
    static constexpr int kTile = 16 * NW;                  // tokens
    static constexpr int kK = kTile * D / 2;               // bytes: codes of K
    static constexpr int kV = kTile * D * 2;               // V
    static constexpr int kS = kTile * D / 32;              // scale bytes of K, then of V
    static constexpr int kBytes = kK + kV + 2 * kS;
    static constexpr int kSlots = 4096;                    // tokens whose slots the workgroup holds
    static constexpr int kLds = 2 * kBytes + kSlots * 4 + 16;
    static constexpr int kKLoads = kTile * D / 32;         // 16-byte chunks of K
    static constexpr int kVLoads = kTile / 4 * (D / 8);    // 4 tokens x 8 dimensions of V
    static constexpr int kSLoads = 2 * kTile;              // scale runs of K and of V
    static constexpr int kKPer = (kKLoads + kThreads - 1) / kThreads;
    static constexpr int kVPer = (kVLoads + kThreads - 1) / kThreads;
};
// Byte of a 16-byte chunk of K's codes, and of one of V's row of tokens: turned
// so that 16 lanes beside each other meet all banks.
template <int D>
DEV int mk_place(int tok, int chunk) {
    constexpr int kChunks = D / 32, kRows256 = 16 / kChunks;
    return tok * (D / 2) + (chunk ^ ((tok / kRows256) & (kChunks - 1))) * 16;
}
template <int TILE>
DEV int mv_place(int dim, int chunk) {
    const int turn = TILE == 128 ? (dim ^ (dim >> 4)) & 15 : ((dim >> 1) ^ (dim >> 4)) & 7;
    return dim * (2 * TILE) + (chunk ^ turn) * 16;
}
typedef float v16f __attribute__((ext_vector_type(16)));
DEV v16f mfma_mx32(v4u a, uint32_t sa, v8i b, uint32_t sb, v16f c) {
    const v8i a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b, c, kFp4, kFp8, 0, (int)sa, 0, (int)sb);
}
template <class E>
DEV v16f mfma32(v4u a, v4u b, v16f c) {
    typedef typename Vec<E>::x8 x8;
    if constexpr (__is_same(E, __bf16))
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}

template <class E, int D, int NW>
__global__ __launch_bounds__(64 * NW, D == 256 ? 1 : 2) void many_rows_kernel(AttnParams p) {
    typedef Many<D, NW> M;
    constexpr int kTerms = __is_same(E, __bf16) ? 2 : 3;
    constexpr int kRuns = D / 64, kDt = D / 32, kRowsWg = 32 * NW;
    typedef typename Vec<E>::x8 x8;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // The last rows, which see the longest context, come first.
    const int64_t units = (int64_t)p.sequences * p.kv_heads * p.splits;
    const Job job = job_of(blockIdx.x, units, p.tiles);
    if (job.unit >= units) return;
    const int tile = p.tiles - 1 - job.inner;
    const int split = (int)(job.unit % p.splits), h = (int)(job.unit / p.splits % p.kv_heads);
    const int b = (int)(job.unit / p.splits / p.kv_heads);

    const Rows rows = rows_of(p, b);
    const int64_t q0 = rows.q0, nq = rows.nq;
    const int shown = rows.shown;
    const int first_row = tile * kRowsWg;
    if (shown <= 0 || first_row / p.group >= shown) return;
    const int64_t held = p.table_width << p.page_shift;
    const int ctx = p.pages > 0 ? (int)min((int64_t)max(p.ctx_len[b], 0), held) : 0;
    const int r = first_row + 32 * wave + col;
    const int qi = r / p.group, qg = r - qi * p.group;
    const bool live = qi < shown;
    const int64_t row = q0 + qi;
    const int hq = h * p.group + qg;
    // last token that this lane's row sees; that all rows of the wave see; tokens that concern the workgroup
    const int last = !live ? -1 : p.causal ? (int)(ctx - nq + qi) : ctx - 1;
    const int all_last = (int)max((int64_t)-1, p.causal ? ctx - nq + (first_row + 32 * wave) / p.group : (int64_t)ctx - 1);
    // (no row sees less than another where it is not causal)
    const int wg_last = p.causal ? (int)max((int64_t)-1, ctx - nq + first_row / p.group) : 0x7FFFFFFF;
    const int wave_last_q = min((first_row + 32 * wave + 31) / p.group, shown - 1);
    const int wave_last = (first_row + 32 * wave) / p.group >= shown ? -1
                          : p.causal ? (int)max((int64_t)-1, ctx - nq + wave_last_q) : ctx - 1;   // that any row of the wave sees
    const int qi_last = min((first_row + kRowsWg - 1) / p.group, shown - 1);
    const int end = (int)max((int64_t)0, p.causal ? ctx - nq + qi_last + 1 : (int64_t)ctx);
    const int64_t lo = (int64_t)split * p.chunk;
    const int begin = (int)min(lo, (int64_t)end), stop = (int)min(lo + p.chunk, (int64_t)end);
    const float scale2 = fabsf(p.scale2);
    const uint32_t record = (uint32_t)p.record;
    const int32_t* table = p.block_table + (int64_t)b * p.table_width;
    const int page_mask = (1 << p.page_shift) - 1;
    int32_t* const slots = reinterpret_cast<int32_t*>(lds + 2 * M::kBytes);
    uint32_t* const nan_flag = reinterpret_cast<uint32_t*>(lds + 2 * M::kBytes + M::kSlots * 4);   // some value is NaN

    // What this thread moves of a tile.
    v4u kreg[M::kKPer];
    uint32_t vreg[M::kVPer][4], vsreg[M::kVPer][4];
    Codes<D / 32> sreg;
    uint32_t vthere[M::kVPer];
    auto fetch = [&](int t_lds) {
#pragma unroll
        for (int c = 0; c < M::kKPer; ++c) {
            const int i = threadIdx.x + c * M::kThreads;
            if (M::kKLoads >= M::kThreads || i < M::kKLoads) {
                const uint32_t slot = (uint32_t)max(slots[t_lds + i / (D / 32)], 0);
                kreg[c] = load16(p.cache + (uint64_t)slot * record + (uint32_t)(h * (D / 2) + (i % (D / 32)) * 16));
            }
        }
#pragma unroll
        for (int c = 0; c < M::kVPer; ++c) {
            const int i = threadIdx.x + c * M::kThreads;
            if (M::kVLoads >= M::kThreads || i < M::kVLoads) {
                const int tg4 = i / (D / 8), dg = i % (D / 8);
                const int4 s4 = *reinterpret_cast<const int4*>(slots + t_lds + 4 * tg4);
                const int ss[4] = {s4.x, s4.y, s4.z, s4.w};
                vthere[c] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint8_t* rec = p.cache + (uint64_t)(uint32_t)max(ss[j], 0) * record;
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)((p.kv_heads + h) * (D / 2) + dg * 4));
                    const uint32_t e = rec[(uint32_t)(p.kv_heads * D + (p.kv_heads + h) * (D / 32) + dg / 4)];
                    vreg[c][j] = w;
                    vsreg[c][j] = e;
                    vthere[c] |= ss[j] >= 0 ? 1u << j : 0u;
                }
            }
        }
        if (threadIdx.x < M::kSLoads) {
            const int v = threadIdx.x / M::kTile;
            const uint32_t slot = (uint32_t)max(slots[t_lds + threadIdx.x % M::kTile], 0);
            sreg = load_codes<D / 32>(p.cache + (uint64_t)slot * record +
                                      (uint32_t)(p.kv_heads * D + (v * p.kv_heads + h) * (D / 32)));
        }
    };
    // The first scale byte that counts as NaN in the tile whose first token is
    // t: where some row does not see all of its tokens, that of values which are
    // infinite in the 16-bit type (weight zero times infinity is not zero).
    auto first_bad = [&](int t) { return t > wg_last - (M::kTile - 1) ? kOver<E> : 255u; };
    auto stage = [&](int buf, int t) {   // the tile of first token t
        const uint32_t bad_from = first_bad(t);
        uint8_t* base = lds + buf * M::kBytes;
#pragma unroll
        for (int c = 0; c < M::kKPer; ++c) {
            const int i = threadIdx.x + c * M::kThreads;
            if (M::kKLoads >= M::kThreads || i < M::kKLoads)
                *reinterpret_cast<v4u*>(base + mk_place<D>(i / (D / 32), i % (D / 32))) = kreg[c];
        }
        bool bad = false;
#pragma unroll
        for (int c = 0; c < M::kVPer; ++c) {
            const int i = threadIdx.x + c * M::kThreads;
            if (M::kVLoads >= M::kThreads || i < M::kVLoads) {
                const int tg4 = i / (D / 8), dg = i % (D / 8);
                // four tokens from 4 tg4: half-chunk (tg4 >> 1) & 1 of chunk 2 s + half
                const int chunk = (tg4 >> 3) * 4 + ((tg4 >> 2) & 1) * 2 + (tg4 & 1), upper = (tg4 >> 1) & 1;
                float sc[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // tokens that are not there, and NaN blocks (their rows get NaN in `use`), are zeros
                    const bool here = (vthere[c] >> j) & 1, nan = vsreg[c][j] >= bad_from;
                    bad |= here && nan;
                    if (!here || nan) vreg[c][j] = 0u, vsreg[c][j] = 127u;
                    sc[j] = scale_of(vsreg[c][j]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t u[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[j] = unpack<E>(vreg[c][j], sc[j], k);
                    uint8_t* at = base + M::kK + upper * 8;
                    *reinterpret_cast<v2u*>(at + mv_place<M::kTile>(8 * dg + 2 * k, chunk)) =
                        v2u{__builtin_amdgcn_perm(u[1], u[0], 0x05040100u), __builtin_amdgcn_perm(u[3], u[2], 0x05040100u)};
                    *reinterpret_cast<v2u*>(at + mv_place<M::kTile>(8 * dg + 2 * k + 1, chunk)) =
                        v2u{__builtin_amdgcn_perm(u[1], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[2], 0x07060302u)};
                }
            }
        }
        if (bad) *nan_flag = 1u;
        if (threadIdx.x < M::kSLoads) {
            uint8_t* at = base + M::kK + M::kV + threadIdx.x * (D / 32);
            if constexpr (D == 64)
                *reinterpret_cast<uint16_t*>(at) = (uint16_t)sreg.w[0];
            else if constexpr (D == 128)
                *reinterpret_cast<uint32_t*>(at) = sreg.w[0];
            else
                *reinterpret_cast<v2u*>(at) = v2u{sreg.w[0], sreg.w[1]};
        }
    };

    // Queries: of dimensions 64 c + 16 half + (0 .. 15) and 32 more, per term.
    v8i qf[kRuns][kTerms];
    uint32_t qs[kRuns];   // scale of dimensions 64 c + 32 half ..
    auto load_queries = [&]() {
        const E* q = live ? static_cast<const E*>(p.q) + row * p.qt + hq * p.qh : nullptr;
        const float sign = p.scale2 < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            float x[2][16];
            uint32_t m[2] = {0, 0};
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x8 v = {};
                    if (q) v = *reinterpret_cast<const x8*>(q + 64 * c + 32 * g + 16 * half + 8 * i);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[g][8 * i + j] = (float)v[j];
                        m[g] = max(m[g], __float_as_uint((float)v[j]) & 0x7FFFFFFFu);
                    }
                }
            uint32_t byte[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                m[g] = max(m[g], (uint32_t)__shfl_xor((int)m[g], 32, 64));
                const int e = (int)(m[g] >> 23);
                byte[g] = e == 255 ? 255u : (uint32_t)max(e - 7, 16);
                const float inv = e == 255 ? 0.f : __uint_as_float((254u - byte[g]) << 23) * sign;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[g][i] = e == 255 ? 0.f : x[g][i] * inv;
            }
            qs[c] = half ? byte[1] : byte[0];
#pragma unroll
            for (int t = 0; t < kTerms; ++t) {
                split16(x[0], qf[c][t], 0);
                split16(x[1], qf[c][t], 4);
            }
        }
    };

    float m = -INFINITY, base = 0.f, sum = 0.f;
    v16f o[kDt];
#pragma unroll
    for (int n = 0; n < kDt; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][i] = 0.f;

    uint32_t nan_blocks = 0;   // bit n: the row sees a value that is NaN in dimensions 32 n ..
    // Where the lane reads K (token col) and V (dimension col): what varies is
    // added or, inside a turned row, flipped.
    const int k_row = mk_place<D>(col, half);
    const int v_row = col * (2 * M::kTile), v_turn = mv_place<M::kTile>(col, half) - v_row;
    // 32 tokens from t0, at token `tok` of the tile in `buf`; bad_from: the tile's first_bad.
    auto use = [&](int buf, int tok, int t0, uint32_t there, uint32_t bad_from) {
        const uint8_t* kb = lds + buf * M::kBytes;
        const uint8_t* vb = kb + M::kK;
        const uint8_t* sb = vb + M::kV + (tok + col) * (D / 32);
        v16f sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kRuns; ++c) {
            const v4u k = *reinterpret_cast<const v4u*>(kb + tok * (D / 2) + (k_row ^ (32 * c)));
            const uint32_t ks = sb[2 * c + half];
#pragma unroll
            for (int t = kTerms - 1; t >= 0; --t)
                sc = mfma_mx32(k, ks, qf[c][t], qs[c] == 255 ? 255u : qs[c] - 4u * t, sc);
        }
        const bool full = there == 0xFFFFFFFFu && t0 + 31 <= all_last;   // wave-uniform
        uint32_t seen = 0;   // bit i: this row sees token 8 (i / 4) + 4 half + i % 4
        if (!full) {
            int half_now = half;
            asm("" : "+v"(half_now));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = 8 * (i >> 2) + 4 * half_now + (i & 3);
                const bool see = ((there >> n) & 1) && t0 + n <= last;
                seen |= see ? 1u << i : 0u;
                if (!see) sc[i] = -INFINITY;
            }
        }
        float top = max3(sc[0], sc[1], sc[2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) top = max3(top, sc[i], sc[i + 1]);
        top = max2(top, sc[15]);
        if (__any(top > m)) {
            const float m_new = fmaxf(m, max_halves(top));
            const float keep = m_new == m || m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * scale2);
            m = m_new;
            base = base_of<E>(m, scale2);
            sum *= keep;
#pragma unroll
            for (int n = 0; n < kDt; ++n) o[n] *= keep;
        }
        float w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = weight_of<E>(sc[i], scale2, base);
        if (!full) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = (seen >> i) & 1 ? w[i] : 0.f;
        }
        float part[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i] = (w[4 * i] + w[4 * i + 1]) + (w[4 * i + 2] + w[4 * i + 3]);
        sum += (part[0] + part[1]) + (part[2] + part[3]);
        v4u pf[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) pf[s][j] = pack2<E>(w[8 * s + 2 * j], w[8 * s + 2 * j + 1]);
        if (__builtin_amdgcn_readfirstlane(*nan_flag)) {
            // Some value block so far is NaN. Its codes were taken as zeros,
            // because a row that does not see it has weight zero, and NaN times
            // zero is not; the rows that see it remember its dimensions.
            const uint8_t* vsb = vb + M::kV + M::kS + tok * (D / 32);
#pragma unroll 1
            for (int t = 0; t < 32; ++t) {
                uint32_t nan = 0;
#pragma unroll
                for (int n = 0; n < D / 32; ++n) nan |= vsb[t * (D / 32) + n] >= bad_from ? 1u << n : 0u;
                nan_blocks |= ((there >> t) & 1) != 0 && t0 + t <= last ? nan : 0u;
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < kDt; ++n) {
                const v4u a = *reinterpret_cast<const v4u*>(vb + v_row + n * (64 * M::kTile) + ((v_turn ^ (2 * tok)) ^ (32 * ((n ^ s) & 3))));
                o[n] = mfma32<E>(a, pf[s], o[n]);
            }
    };

    if (threadIdx.x == 0) *nan_flag = 0u;
    for (int64_t from = begin; from < stop; from += M::kSlots) {
        const int piece = (int)from;
        const int fill = min(stop - piece, M::kSlots), padded = (fill + M::kTile - 1) / M::kTile * M::kTile;
        lds_barrier();
        for (int i = threadIdx.x; i < padded; i += M::kThreads) {
            int slot = -1;
            if (i < fill) {
                const int page = table[(piece + i) >> p.page_shift];
                if ((uint32_t)page < (uint32_t)p.pages) slot = (page << p.page_shift) + ((piece + i) & page_mask);
            }
            slots[i] = slot;
        }
        lds_barrier();
        fetch(0);
        if (piece == begin) load_queries();
        stage(0, piece);
        fetch(min(M::kTile, padded - M::kTile));
        lds_barrier();
        int buf = 0;
        for (int t = 0; t < padded; t += M::kTile) {
            stage(buf ^ 1, step_at(piece, t + M::kTile));
            fetch(min(t + 2 * M::kTile, padded - M::kTile));
#pragma unroll 1
            for (int s = 0; s < M::kTile; s += 32) {
                const int t0 = step_at(piece, t + s);
                if (t0 > wave_last) break;
                const uint32_t there = (uint32_t)__ballot(slots[t + s + col] >= 0);
                use(buf, s, t0, there, first_bad(step_at(piece, t)));
            }
            lds_barrier();
            buf ^= 1;
        }
    }
    sum += __shfl_xor(sum, 32, 64);
    if constexpr (!__is_same(E, __bf16)) {
        sum *= kDown;
#pragma unroll
        for (int n = 0; n < kDt; ++n) o[n] *= kDown;
    }
    if (!live) return;
    if (nan_blocks) {
#pragma unroll
        for (int n = 0; n < kDt; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[n][i] += (nan_blocks >> n) & 1 ? __builtin_nanf("") : 0.f;
    }
    const int64_t at = row * p.q_heads + hq;
    const float m2 = m == -INFINITY ? m : m * scale2;
    // lane: row col, dimensions 32 n + 8 b + 4 half + (0 .. 3)
    if (p.splits > 1) {
        const int64_t part = (((int64_t)b * p.splits + split) * p.max_q + qi) * p.q_heads + hq;
        if (half == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * part) = float2{m2, sum};
        if (sum == 0.f) return;
        float* po = p.part_o + part * D + 4 * half;
#pragma unroll
        for (int n = 0; n < kDt; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<v4f*>(po + 32 * n + 8 * g) = v4f{o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2], o[n][4 * g + 3]};
        return;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;   // NaN stays
    if (p.lse && half == 0) p.lse[at] = sum == 0.f ? -INFINITY : (m2 + log2f(sum)) * kLn2;
    uint16_t* out = static_cast<uint16_t*>(p.out) + at * D + 4 * half;
#pragma unroll
    for (int n = 0; n < kDt; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<v2u*>(out + 32 * n + 8 * g) = v2u{pack2<E>(o[n][4 * g] * inv, o[n][4 * g + 1] * inv),
                                                             pack2<E>(o[n][4 * g + 2] * inv, o[n][4 * g + 3] * inv)};
}

// One workgroup per served query row and head: its splits joined in a fixed
// order, `kAt` at a time. The weights are made first, so that the loads of the
// parts wait for nothing.
template <class E, int D>
__global__ __launch_bounds__(gvr_kv4::kJoinThreads) void combine_kernel(AttnParams p) {
    constexpr int kPer = D / 4;            // threads of a split: four dimensions each
    constexpr int kAt = 256 / kPer;        // splits at a time
    __shared__ float4 acc_l[256];
    __shared__ float weight_l[kMaxSplits], red_l[8];
    const int hq = (int)(blockIdx.x % (uint32_t)p.q_heads);
    const int job = (int)(blockIdx.x / (uint32_t)p.q_heads), b = job / p.max_q, i = job % p.max_q;
    const Rows r = rows_of(p, b);
    if (i >= r.shown) return;
    const int64_t at = (r.q0 + i) * p.q_heads + hq;
    const int2 units = p.balanced ? p.units_of[b] : int2{b * p.splits, p.splits};
    const int splits = units.y;
    if (splits == 1) return;               // the unit wrote the result
    const int64_t step = (int64_t)p.max_q * p.q_heads, first_part = (units.x * (int64_t)p.max_q + i) * p.q_heads + hq;
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + first_part;
    const int lane = threadIdx.x % kPer, first = threadIdx.x / kPer;
    const float4* po = reinterpret_cast<const float4*>(p.part_o + first_part * D) + lane;
    const float4 x0 = po[min(first, splits - 1) * step * kPer];   // (with the weights' loads)
    float m = -INFINITY;
    for (int s = threadIdx.x; s < splits; s += 256) {
        const float2 v = ml[s * step];
        m = fmaxf(m, v.y == 0.f ? -INFINITY : v.x);
    }
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if ((threadIdx.x & 63) == 0) red_l[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red_l[0], red_l[1]), fmaxf(red_l[2], red_l[3]));
    const float base = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    for (int s = threadIdx.x; s < splits; s += 256) {
        const float2 v = ml[s * step];
        const bool wrote = v.y != 0.f;     // (else it saw nothing)
        const float w = wrote ? __builtin_amdgcn_exp2f(v.x - base) : 0.f;
        weight_l[s] = wrote ? w : -1.f;
        sum += w * v.y;
    }
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((threadIdx.x & 63) == 0) red_l[4 + (threadIdx.x >> 6)] = sum;
    __syncthreads();
    sum = (red_l[4] + red_l[5]) + (red_l[6] + red_l[7]);
    float4 acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float w, const float4& x) {
        // What was not written may be anything. A part whose weight is zero counts:
        // a NaN that its row sees stays one, as without splits.
        const bool seen = !(w < 0.f);
        acc.x += seen ? w * x.x : 0.f, acc.y += seen ? w * x.y : 0.f;
        acc.z += seen ? w * x.z : 0.f, acc.w += seen ? w * x.w : 0.f;
    };
    if (first < splits) add(weight_l[first], x0);
#pragma unroll 8
    for (int s = first + kAt; s < splits; s += kAt) add(weight_l[s], po[s * step * kPer]);
    acc_l[threadIdx.x] = acc;
    __syncthreads();
    if (first != 0) return;
    acc = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kAt; ++s) {
        const float4 x = acc_l[s * kPer + lane];
        acc.x += x.x, acc.y += x.y, acc.z += x.z, acc.w += x.w;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (p.lse && lane == 0) p.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
    uint2* out = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at * D) + lane;
    *out = uint2{pack2<E>(acc.x * inv, acc.y * inv), pack2<E>(acc.z * inv, acc.w * inv)};
}

template <class E, int D>
gvr_status launch(const AttnParams& p, int64_t jobs, void* stream) {
    if (p.many) {
        typedef Many<D, D == 256 ? 4 : 8> M;
        hipLaunchKernelGGL((many_rows_kernel<E, D, D == 256 ? 4 : 8>), dim3((unsigned)jobs), dim3(M::kThreads), M::kLds,
                           (hipStream_t)stream, p);
    } else {
        const int rows = p.row_tiles;
        const int join = p.tw_shift ? gvr_kv4::kWaves / 2 * rows * (D / 16 * 1024 + 512) : 0;   // bytes of the waves' join
        const int queries = (rows * Query<E, D>::kRuns * Query<E, D>::kPer * 2048) << p.hw_shift;
        const int lds = max(join, WaveLds<D>::kLds + queries);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)jobs), dim3(kThreads), lds, (hipStream_t)stream, p);
        };
        if constexpr (D != 256)
            rows == 2 ? go(few_rows_kernel<E, D, 2>) : go(few_rows_kernel<E, D, 1>);
        else
            go(few_rows_kernel<E, D, 1>);
    }
    if (hipGetLastError() != hipSuccess) return GVR_ERR_HIP;
    if (p.splits > 1 || p.balanced) {
        hipLaunchKernelGGL((combine_kernel<E, D>), dim3((unsigned)((int64_t)p.sequences * p.max_q * p.q_heads)),
                           dim3(gvr_kv4::kJoinThreads), 0, (hipStream_t)stream, p);
        if (hipGetLastError() != hipSuccess) return GVR_ERR_HIP;
    }
    return GVR_OK;
}
template <class E>
gvr_status launch_d(const AttnParams& p, int64_t jobs, int D, void* stream) {
    return D == 64 ? launch<E, 64>(p, jobs, stream) : D == 128 ? launch<E, 128>(p, jobs, stream) : launch<E, 256>(p, jobs, stream);
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
    if (a.T == 0 || a.sequences == 0 || (a.q_start && a.max_q == 0)) return GVR_OK;
    if (!a.q || !a.out || !a.ctx_len || (!a.block_table && a.table_width > 0)) return GVR_ERR_INVALID_ARG;
    if (((uintptr_t)a.q | (uintptr_t)a.out) & 15) return GVR_ERR_INVALID_ARG;
    const gvr_kv4::AttnPlan plan = gvr_kv4::plan_attention(*cache, a, ws_bytes);
    if (plan.jobs > gvr_kv4::kMaxThreads / plan.threads) return GVR_ERR_TOO_LONG;
    AttnParams p;
    p.cache = cache->data;
    p.q = a.q, p.qt = a.q_token_stride, p.qh = a.q_head_stride;
    p.out = a.out, p.lse = a.lse;
    p.block_table = a.block_table, p.ctx_len = a.ctx_len, p.q_start = a.q_start, p.selection = a.selection;
    p.table_width = a.table_width, p.pages = (int32_t)cache->pages, p.T = a.T;
    p.record = gvr_kv4::record_bytes(cache->kv_heads, cache->head_dim);
    p.page_shift = gvr_kv4::log2_of(cache->page_size);
    p.kv_heads = cache->kv_heads, p.q_heads = a.q_heads, p.group = a.q_heads / cache->kv_heads;
    p.sequences = a.sequences;
    p.uniform_q = a.q_start ? 0 : (int32_t)(a.T / a.sequences);
    p.max_q = plan.max_q, p.tiles = plan.tiles, p.splits = plan.splits, p.chunk = plan.chunk;
    p.many = plan.many, p.row_tiles = plan.row_tiles;
    p.hw_shift = plan.hw_shift, p.tw_shift = plan.tw_shift;
    p.K = a.K, p.causal = a.causal;
    p.scale2 = a.scale * kLog2e;
    p.balanced = plan.balanced, p.units = plan.units;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + (int64_t)plan.units * plan.max_q * a.q_heads * cache->head_dim;
    p.units_of = reinterpret_cast<int2*>(p.part_ml + (int64_t)plan.units * plan.max_q * a.q_heads * 2);
    return a.dtype == GVR_BF16 ? launch_d<__bf16>(p, plan.jobs, cache->head_dim, stream)
                               : launch_d<_Float16>(p, plan.jobs, cache->head_dim, stream);
}

}  // extern "C"
