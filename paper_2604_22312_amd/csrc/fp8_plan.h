// fp8_plan.h -- argument checks and launch plans of the 8-bit matrices: making
// them and multiplying them. Plain C++ with no HIP dependency, so the library
// and a sanitizer build on the CPU compile the same code.
#ifndef GVR_FP8_PLAN_H
#define GVR_FP8_PLAN_H

#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "gvr_fp8.h"
#include "rotary_plan.h"

namespace gvr_fp8 {

using gvr_rot::kMaxCount;

constexpr int kGroup = 128;       // elements that share a scale
constexpr int kBlock = 256;       // threads of the quantising kernels
constexpr int kMaxHead = 1 << 20; // elements of a head, and heads

inline int64_t groups_of(int64_t n) { return (n + kGroup - 1) / kGroup; }

// Division of 32-bit numbers below 2^31 by a number that the launch knows: n / d is
// the upper half of n * mul, shifted (mul = ceil(2^(32 + shift) / d), shift the bits of
// d - 1, fits 33 bits; its upper bit is added by hand).
struct Divisor {
    uint32_t d, mul, shift;
};
inline Divisor divisor(uint32_t d) {
    Divisor r = {d, 0, 0};
    while (((uint64_t)1 << r.shift) < d) ++r.shift;
    r.mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << r.shift) - d)) / d + 1);
    return r;
}
inline uint32_t quotient(uint32_t n, const Divisor& r) {
    return (uint32_t)((((uint64_t)n * r.mul >> 32) + n) >> r.shift);
}

// --- heads: a thread takes 8 elements of a block of 128, or 16
struct HeadsPlan {
    int64_t tokens, blocks, rows;   // of a launch row (blockIdx.y), workgroups in x, launch rows
};
inline HeadsPlan plan_heads(int64_t T, int64_t lanes_per_token) {
    HeadsPlan p;
    p.tokens = kMaxCount / lanes_per_token;
    if (p.tokens > T) p.tokens = T;
    if (p.tokens < 1) p.tokens = 1;
    p.blocks = (p.tokens * lanes_per_token + kBlock - 1) / kBlock;
    p.rows = (T + p.tokens - 1) / p.tokens;
    return p;
}

inline gvr_status check_heads(const gvr_heads* x, int dtype, int64_t T, int H, int D, const int32_t* positions,
                              const gvr_rope_cs* cs, const gvr_fp8_heads* out, const int64_t* slots, int64_t rows,
                              int flags) {
    const int size = gvr_rot::dtype_size(dtype);
    if (!x || !out || size == 0 || T < 0 || H < 0 || D < 1 || rows < 0 || (flags & ~GVR_FP8_POW2)) return GVR_ERR_INVALID_ARG;
    if (T > kMaxCount || rows > kMaxCount || H > kMaxHead || D > kMaxHead) return GVR_ERR_TOO_LONG;
    if (((uintptr_t)x->data & (size - 1)) || ((uintptr_t)out->scale & 3) || ((uintptr_t)slots & 7)) return GVR_ERR_INVALID_ARG;
    if (cs) {
        const gvr_status st = gvr_rot::check_cs(*cs, D, GVR_ROPE_INTERLEAVED);
        if (st != GVR_OK) return st;
        if (T > 0 && H > 0 && (!positions || ((uintptr_t)positions & 3))) return GVR_ERR_INVALID_ARG;
    }
    if (T == 0 || H == 0) return GVR_OK;
    if (!x->data || !out->codes || !out->scale) return GVR_ERR_INVALID_ARG;
    if (!slots && rows < T) return GVR_ERR_INVALID_ARG;
    const int64_t lanes = (int64_t)H * groups_of(D) * 16;
    if (lanes > kMaxCount || plan_heads(T, lanes).rows > gvr_rot::kMaxRows) return GVR_ERR_TOO_LONG;
    return GVR_OK;
}

// --- matrices: a workgroup takes 128 x 128 elements
inline gvr_status check_matrix(const gvr_fp8_matrix& m, int rows_per_scale, bool need) {
    if (m.reserved != 0 || m.rows_per_scale != rows_per_scale) return GVR_ERR_INVALID_ARG;
    if (need && (!m.codes || !m.scale)) return GVR_ERR_INVALID_ARG;
    if ((uintptr_t)m.scale & 3) return GVR_ERR_INVALID_ARG;
    return GVR_OK;
}
inline gvr_status check_quantize_matrix(const void* x, int dtype, int64_t R, int64_t C, const gvr_fp8_matrix* straight,
                                        const gvr_fp8_matrix* transposed, int flags) {
    const int size = gvr_rot::dtype_size(dtype);
    if (size == 0 || R < 0 || C < 0 || (flags & ~(GVR_FP8_POW2 | GVR_FP8_SQUARE))) return GVR_ERR_INVALID_ARG;
    const bool need = R > 0 && C > 0;
    for (const gvr_fp8_matrix* m : {straight, transposed})
        if (m) {
            const gvr_status st = check_matrix(*m, flags & GVR_FP8_SQUARE ? kGroup : 1, need);
            if (st != GVR_OK) return st;
        }
    if (R > kMaxCount || C > kMaxCount) return GVR_ERR_TOO_LONG;
    if ((uintptr_t)x & (size - 1)) return GVR_ERR_INVALID_ARG;
    if (!need || (!straight && !transposed)) return GVR_OK;
    if (!x) return GVR_ERR_INVALID_ARG;
    if (groups_of(R) * groups_of(C) >= (1 << 24)) return GVR_ERR_TOO_LONG;   // (a launch has fewer than 2^32 threads)
    return GVR_OK;
}

// --- products
inline gvr_status check_matmul(const gvr_fp8_matrix* a, const gvr_fp8_matrix* b, int64_t M, int64_t N, int64_t K,
                               bool pointers) {
    if (!a || !b || M < 0 || N < 0 || K < 0 || a->rows_per_scale != 1 || !(b->rows_per_scale == 1 || b->rows_per_scale == kGroup))
        return GVR_ERR_INVALID_ARG;
    const bool need = pointers && M > 0 && N > 0 && K > 0;
    const gvr_status sa = check_matrix(*a, 1, need), sb = check_matrix(*b, b->rows_per_scale, need);
    if (sa != GVR_OK || sb != GVR_OK) return GVR_ERR_INVALID_ARG;
    if (M > kMaxCount || N > kMaxCount || K > kMaxCount) return GVR_ERR_TOO_LONG;
    return GVR_OK;
}

constexpr int kTileM = 64, kTileN = 64, kThreads = 256;   // of the kernel that takes any alignment
enum Shape { kAnyShape, kRows, kRowPairs, kRows32, kLow, kNarrow, kSquare, kLarge };
// Rows of A and of B of a workgroup and its threads; and, measured on 256 compute
// units over K = 4096, the microseconds of a step of 128 elements where a unit runs
// one workgroup and where it runs two (0: it holds one), and of a workgroup's begin and end.
struct Tiles {
    int m, n, threads;
    double one, two, ends;
};
inline Tiles tiles_of(Shape s) {
    switch (s) {
        case kRows: return {16, 16, 512, 0, 0, 0};
        case kRowPairs: return {16, 32, 512, 0, 0, 0};
        case kRows32: return {32, 16, 512, 0, 0, 0};
        case kLow: return {64, 128, 256, 0.60, 0.76, 3.5};
        case kNarrow: return {128, 64, 256, 0.60, 0.76, 3.5};
        case kSquare: return {128, 128, 256, 0.87, 1.33, 3.5};
        case kLarge: return {256, 256, 512, 1.60, 0, 8.0};
        default: return {kTileM, kTileN, kThreads, 0, 0, 0};
    }
}
constexpr int64_t kUnits = 256; // compute units

struct MatmulPlan {
    Shape shape;
    int threads;
    int64_t tiles_m, tiles_n, splits, steps_each, band, workgroups;
    size_t workspace;   // bytes of the splits' parts
};

// Rows that 16-byte loads can serve and that 32-bit offsets reach over a tile of
// `rows` of them.
inline bool tile_rows(const gvr_fp8_matrix& m, int rows, int64_t K) {
    return ((uintptr_t)m.codes & 15) == 0 && m.row_stride % 16 == 0 && m.row_stride >= 0 &&
           m.row_stride * rows + K < kMaxCount && m.scale_row_stride >= 0 && m.scale_block_stride >= 0 &&
           m.scale_row_stride < (1 << 20) && m.scale_block_stride < (1 << 28) &&
           (m.scale_row_stride * rows + m.scale_block_stride * groups_of(K)) * 4 < kMaxCount;
}

// Scales that 16-byte loads of four blocks can serve.
inline bool scale_quads(const gvr_fp8_matrix& m, int64_t K, int64_t steps_each) {
    return ((uintptr_t)m.scale & 15) == 0 && m.scale_block_stride == 1 && m.scale_row_stride % 4 == 0 &&
           groups_of(K) % 4 == 0 && K % kGroup == 0 && steps_each % 4 == 0;
}

// The steps of each part of a sum that is split over about n workgroups (scales come
// four at a time), and how many parts that makes.
struct Split {
    int64_t each, parts;
};
inline Split split_of(int64_t steps, int64_t n) {
    Split s;
    s.each = (steps + n - 1) / n;
    if (n > 1) s.each = (s.each + 3) / 4 * 4;
    s.parts = s.each ? (steps + s.each - 1) / s.each : 1;
    return s;
}

// The time that a shape takes, in microseconds: rounds of workgroups, each as long
// as its steps, and where the sum is split the kernel that joins the parts. (Of the
// splits as they are asked for: with those of split_of in their place one plan in sixteen
// differs, and 40 of these products took 827 us together, not 817.)
inline double matmul_time(const Tiles& t, int64_t M, int64_t N, int64_t steps, int64_t splits) {
    const int64_t units = ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n) * splits, each = (steps + splits - 1) / splits;
    const int64_t round = t.two > 0 ? 2 * kUnits : kUnits, whole = units / round, rest = units % round;
    const double full = t.ends + each * (t.two > 0 ? t.two : t.one);
    double us = whole * full + (rest == 0 ? 0 : rest <= kUnits ? t.ends + each * t.one : full);
    if (splits > 1) us += 2.5 + 8.0e-6 * M * N * splits / 4.5;
    return us;
}

// What a shape and a split come to as a launch. The kernels of few rows hold all of A's
// and take a workgroup's rows of B from its number alone, so more tiles along A or a
// split sum would run them past the end of B: a shape that cannot do these sizes is an
// error, and nothing is launched.
inline gvr_status lay_out(Shape shape, int64_t splits, int64_t M, int64_t N, int64_t K, bool wide, MatmulPlan* p) {
    const Tiles t = tiles_of(shape);
    p->shape = shape;
    p->threads = t.threads;
    p->tiles_m = (M + t.m - 1) / t.m;
    p->tiles_n = (N + t.n - 1) / t.n;   // (each at most 2^27)
    if (shape == kRows && p->tiles_n < kUnits) p->threads = 1024;   // (more waves where workgroups are few)
    const Split split = split_of(groups_of(K), splits);
    p->steps_each = split.each;
    p->splits = split.parts;
    p->band = 4;   // (8192 x 8192 x 4096: 243 us, of 2 and 8 246 and 245, of 16 248; 16384 x 8192 x 4096: 467, 485 and 479, 493)
    p->workspace = p->splits > 1 ? (size_t)p->splits * M * N * 4 : 0;
    p->workgroups = p->tiles_m * p->tiles_n * p->splits;
    const bool rows = shape == kRows || shape == kRowPairs || shape == kRows32;
    if ((rows && p->tiles_m != 1) || (shape < kLow && p->splits != 1) || (shape == kLarge && wide)) return GVR_ERR_INVALID_ARG;
    return p->workgroups * p->threads > 0xFFFFFFFFll ? GVR_ERR_TOO_LONG : GVR_OK;
}

inline gvr_status plan_matmul(const gvr_fp8_matrix& a, const gvr_fp8_matrix& b, int64_t M, int64_t N, int64_t K, bool wide,
                              size_t ws_bytes, MatmulPlan* p) {
    const int64_t steps = groups_of(K);
    int64_t splits = 1;
    Shape shape = kAnyShape;
    if (tile_rows(a, 256, K) && tile_rows(b, 256, K)) {
        // Few rows of A: the kernels without tiles (the times are at them), with two tiles of B's rows to a workgroup
        // where that still gives one to each compute unit (1 x 8192 x 4096: 8.0 us, with one 8.6; 16 x: 9.7, 11.7).
        if (M <= 16 && N <= 1 << 26) {   // (more rows of B: more threads than a launch has)
            shape = N >= 32 * kUnits ? kRowPairs : kRows;
        } else if (M <= 32 && N <= 16 * kUnits) {
            shape = kRows32;
        } else {
            double best = 1e300;
            for (const Shape s : {kLow, kNarrow, kSquare, kLarge})
                for (const int64_t n : {1, 2, 3, 4, 6, 8, 12, 16}) {
                    if (s == kLarge && wide) continue;   // (its sums are on the FP8 matrix cores)
                    const Tiles t = tiles_of(s);
                    // (many workgroups need no splits: the kernel that joins them is launched over few rows)
                    if (n > 1 && (steps < 4 * n || (double)split_of(steps, n).parts * M * N * 4 > (double)ws_bytes ||
                                  ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n) > 4 * kUnits))
                        break;
                    const double us = matmul_time(t, M, N, steps, n);
                    if (us < best) best = us, shape = s, splits = n;
                }
        }
    }
    return lay_out(shape, splits, M, N, K, wide, p);
}

// A product whose rows 16-byte loads cannot serve: its codes are copied to rows that
// they can, in the workspace, if that has room, and the copies are multiplied. Packed
// rows of both, copied and where they are: 1 x 64 x 101 6.1 us and 6.3, 1 x 4096 x 4099
// 15.6 and 41, 128 x 4096 x 4099 25 and 115, 4096 x 4096 x 101 16.8 and 70, 4096 x 4096 x
// 4099 83 and 1760.
struct Product {
    MatmulPlan plan;
    bool copied[2];       // A, B
    int64_t row_stride;   // of the copies
    size_t at[2], parts;  // where the copies and the splits' parts begin
    size_t workspace;     // bytes in all
};

inline bool wide_rows(const gvr_fp8_matrix& m, int64_t K) {
    return ((uintptr_t)m.codes & 15) == 0 && m.row_stride % 16 == 0 && m.row_stride >= 0 && m.row_stride * 256 + K < kMaxCount;
}

inline gvr_status plan_product(const gvr_fp8_matrix& a, const gvr_fp8_matrix& b, int64_t M, int64_t N, int64_t K, bool wide,
                               size_t ws_bytes, Product* p) {
    const int64_t rows[2] = {M, N}, chunks = (K + 15) / 16;
    gvr_fp8_matrix m[2] = {a, b};
    p->row_stride = 16 * chunks;
    p->parts = 0;
    bool any = false, room = K > 0;
    int64_t items = 0;
    for (int i = 0; i < 2; ++i) {
        if (rows[i] <= 1) m[i].row_stride = 0;   // (there is no next row)
        p->copied[i] = !wide_rows(m[i], K);
        p->at[i] = p->parts;
        if (!p->copied[i]) continue;
        any = true;
        room = room && rows[i] < (kMaxCount - items) / chunks;   // (the copying kernel counts in 32 bits)
        if (!room) break;
        items += rows[i] * chunks;
        p->parts += ((size_t)rows[i] * p->row_stride + 255) / 256 * 256;
        m[i].codes = nullptr, m[i].row_stride = p->row_stride;
    }
    if (!any || (room && p->parts <= ws_bytes)) {
        const gvr_status st = plan_matmul(m[0], m[1], M, N, K, wide, ws_bytes - p->parts, &p->plan);
        p->workspace = p->parts + p->plan.workspace;
        if (!any || (st == GVR_OK && p->plan.shape != kAnyShape)) return st;
    }
    p->copied[0] = p->copied[1] = false;
    p->parts = 0;
    const gvr_status st = plan_matmul(a, b, M, N, K, wide, ws_bytes, &p->plan);
    p->workspace = p->plan.workspace;
    return st;
}

}  // namespace gvr_fp8

#endif  // GVR_FP8_PLAN_H
