// fp8_codes.h -- scales and E4M3 codes of a block of elements, for the kernels
// that quantise.
//
// A code is the nearest to 448 x / m (ties to even), m the block's largest
// magnitude. gfx950's conversion rounds a float32 quotient so; the quotient
// itself is x times 448 / m, off by at most two units in the last place, which
// matters only beside the border of two codes. Quotients of short numbers often
// lie on one exactly (bfloat16 elements under m = 1.75 * 2^k: one in sixteen), so
// an element within 8 units of a border is divided in float64, and that quotient
// is rounded to float32 towards odd, which no border is, before it is converted.
// Scales that are powers of two need none of it.
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

// Scale of a block, what its elements are multiplied with, and the magnitude of
// code 448 (0 where no element needs the float64 quotient).
struct Scale {
    float scale, unit, full;
    bool nan;
};
// bits: of the block's largest magnitude (infinities and NaN included).
DEV Scale scale_of(uint32_t bits, bool pow2) {
    Scale s;
    s.nan = bits >= 0x7F800000u;
    const float m = fmaxf(__uint_as_float(bits), kMost * 0x1p-126f);
    if (pow2) {   // m = f 2^e, 448 = 1.75 * 2^8
        const uint32_t b = __float_as_uint(m);
        const uint32_t e = (b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        s.scale = __uint_as_float(e << 23);
        s.unit = __uint_as_float((254u - e) << 23);
        s.full = 0.f;
    } else {
        s.scale = m / kMost;
        s.unit = kMost / m;
        s.full = m;
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
// Largest over the 16 lanes of a row.
DEV uint32_t row_largest(uint32_t m) {
    using namespace gvr_dev;
    m = max(m, (uint32_t)dpp_i<kQuadSwap1>(0, (int)m));
    m = max(m, (uint32_t)dpp_i<kQuadSwap2>(0, (int)m));
    m = max(m, (uint32_t)dpp_i<kRowHalfMirror>(0, (int)m));
    return max(m, (uint32_t)dpp_i<kRowMirror>(0, (int)m));
}

// Whether y is within 8 units of a border: borders are odd multiples of half a
// step, the middle of the 20 bits that the conversion drops; below 2^-6, where
// steps stay 2^-9, adding 2^-6 brings them there.
DEV bool beside_border(float y) {
    float z = fabsf(y);
    z = z < 0x1p-6f ? z + 0x1p-6f : z;
    return ((__float_as_uint(z) + 0x80000u + 8u) & 0xFFFFFu) <= 16u;
}
// 448 x / full, rounded to float32 towards odd.
DEV float exact_quotient(float x, float full) {
    const double q = (double)x * 448.0 / (double)full;
    const float r = (float)q;
    if ((double)r == q) return r;
    uint32_t b = __float_as_uint(r);
    if (fabs((double)r) > fabs(q)) --b;
    return __uint_as_float(b | 1u);
}

// Eight codes.
DEV uint2 codes_of(f8 x, const Scale& s) {
    f8 y;
    bool beside = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = x[i] * s.unit;
        beside |= beside_border(y[i]);
    }
    if (beside && s.full != 0.f) {
#pragma unroll 1
        for (int i = 0; i < 8; ++i) y[i] = exact_quotient(x[i], s.full);
    }
    uint2 c;
    c.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c.x, true);
    c.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    c.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], c.y, true);
    if (s.nan) c.x = c.y = kNan4;
    return c;
}

}  // namespace gvr_fp8c

#endif  // GVR_FP8_CODES_H
