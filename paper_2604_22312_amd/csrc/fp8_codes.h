// fp8_codes.h -- scales and E4M3 codes of a block of elements, for the kernels
// that quantise.
//
// A code is the nearest to 448 x / m (ties to even), m the block's largest
// magnitude. gfx950's conversion rounds a float32 quotient so, but x times 448 / m is
// the quotient only to within 2^-22 of it, which matters beside the border of two
// codes; and quotients of short numbers often lie on one exactly (bfloat16: m of one
// block in seven is a multiple of 7 / 8 of its power of two, and then about one element
// in sixteen lies on a border).
//
// The factor 448 / m is itself within 3 * 2^-24, from the hardware's reciprocal (three
// IEEE divisions a block instead: 4096 x 4096 bfloat16 in both directions 26.2 us, not
// 22.0).
//
// Elements of 16 bits: 448 x is exact, so one correction by the remainder, y + (448 x -
// y m) / m, is the quotient where that fits float32, which it does on every border;
// beside one the quotient is at least 2^-17 of itself away, more than any error left.
//
// Elements of 32 bits: x is multiplied with a little less and a little more (2^-21 of it)
// than 448 / m. Where both products have the same code, the quotient between them has it
// too; elsewhere (one element of 2^16) 448 x is compared with the border times m, exactly.
// This for bfloat16 too: 4096 x 4096 in both directions 27.0 us against 23.8 (with
// the divisions).
#ifndef GVR_FP8_CODES_H
#define GVR_FP8_CODES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem_ops.h"
#include "wave_ops.h"

namespace gvr_fp8c {

using gvr_elem::f8;

constexpr float kMost = 448.f;
constexpr uint32_t kNan4 = 0x7F7F7F7Fu;   // four NaN codes

// Scale of a block, 448 / m, and m, as `part` times a power of two (of `sized`) that
// keeps products with it from overflowing and losing bits.
struct Scale {
    float scale, unit, part, size;
    bool nan;
};
// bits: of the block's largest magnitude (infinities and NaN included).
DEV Scale scale_of(uint32_t bits, bool pow2) {
    Scale s;
    s.nan = bits >= 0x7F800000u;
    const float m = fmaxf(__uint_as_float(bits), kMost * 0x1p-126f);
    s.size = m > 1.f ? 0x1p-20f : 0x1p40f;
    if (pow2) {   // m = f 2^e, 448 = 1.75 * 2^8
        const uint32_t b = __float_as_uint(m);
        const uint32_t e = (b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        s.scale = __uint_as_float(e << 23);
        s.unit = __uint_as_float((254u - e) << 23);
        s.part = kMost * (s.scale * s.size);
    } else {
        // m / 448 by its reciprocal and one correction, which rounds it right (checked for every fraction, least exponents
        // included); 448 / m from a reciprocal within one unit, of a number far from either end of the range
        const float q = m * (1.f / kMost);
        s.scale = __fmaf_rn(__fmaf_rn(-q, kMost, m), 1.f / kMost, q);
        s.part = m * s.size;
        s.unit = kMost * s.size * __builtin_amdgcn_rcpf(s.part);
    }
    if (s.nan) s.scale = __uint_as_float(0x7FC00000u);
    return s;
}

DEV uint32_t largest(f8 x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return m;
}
// Largest over LANES (8 or 16) neighbouring lanes.
template <int LANES>
DEV uint32_t row_largest(uint32_t m) {
    using namespace gvr_dev;
    m = max(m, (uint32_t)dpp_i<kQuadSwap1>(0, (int)m));
    m = max(m, (uint32_t)dpp_i<kQuadSwap2>(0, (int)m));
    m = max(m, (uint32_t)dpp_i<kRowHalfMirror>(0, (int)m));
    return LANES == 8 ? m : max(m, (uint32_t)dpp_i<kRowMirror>(0, (int)m));
}

DEV uint2 convert8(f8 y) {
    uint2 c;
    c.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c.x, true);
    c.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    c.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], c.y, true);
    return c;
}

// The code of x, of magnitude code `low` or the one above it: which side of the border
// between them 448 x / m is on. 448 x is held in two parts, and the difference to the
// product of the border, a number of five bits, is exact: they are within 2^-20.
DEV uint32_t settle(uint32_t low, float x, const Scale& s) {
    const float border = 0.5f * (__builtin_amdgcn_cvt_f32_fp8((int)low, 0) + __builtin_amdgcn_cvt_f32_fp8((int)low + 1, 0));
    const float a = fabsf(x) * s.size, hi = kMost * a, lo = __fmaf_rn(kMost, a, -hi);
    const float beyond = __fmaf_rn(border, s.part, -hi) - lo;   // border * m - 448 x
    return beyond < 0.f || (beyond == 0.f && (low & 1)) ? low + 1 : low;
}

// Eight codes; SHORT: of elements that came from 16 bits.
template <bool SHORT>
DEV uint2 codes_of(f8 x, const Scale& s) {
    f8 y;
    uint2 c;
    if constexpr (SHORT) {
        const float to = kMost * s.size, back = s.unit * (s.size < 1.f ? 0x1p20f / kMost : 0x1p-40f / kMost);   // 1 / part
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = x[i] * s.unit;
            y[i] = __fmaf_rn(-__fmaf_rn(q, s.part, -(x[i] * to)), back, q);   // (this way round -0 stays -0)
        }
        c = convert8(y);
    } else {
        const float below = s.unit * (1.f - 0x1p-21f), above = s.unit * (1.f + 0x1p-21f);
        f8 z;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i] * below, z[i] = x[i] * above;
        c = convert8(y);
        const uint2 d = convert8(z);
        if (c.x != d.x || c.y != d.y) {
            // (element by element: few of them are beside a border in any lane)
            const uint32_t off[2] = {c.x ^ d.x, c.y ^ d.y};
            uint32_t r[2] = {c.x, c.y};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t at = 8 * (i & 3);
                if (off[i / 4] >> at & 0xFFu) {
                    const uint32_t low = r[i / 4] >> at & 0x7Fu;
                    r[i / 4] += (settle(low, x[i], s) - low) << at;
                }
            }
            c.x = r[0], c.y = r[1];
        }
    }
    if (s.nan) c.x = c.y = kNan4;
    return c;
}

}  // namespace gvr_fp8c

#endif  // GVR_FP8_CODES_H
