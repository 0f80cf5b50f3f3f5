// elem_ops.h -- loads and stores of eight consecutive elements of a bfloat16,
// float16 or float32 tensor as float32 values, for the rotary and the 4-bit
// cache kernels.
#ifndef GVR_ELEM_OPS_H
#define GVR_ELEM_OPS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#ifndef DEV
#define DEV __device__ __forceinline__
#endif

namespace gvr_elem {

typedef float f8 __attribute__((ext_vector_type(8)));
// (eight float32 would ask for 32-byte alignment; rows promise 16)
template <class E> struct Vec8 { typedef E t __attribute__((ext_vector_type(8), aligned(16))); };
static_assert(alignof(Vec8<float>::t) == 16 && alignof(Vec8<__bf16>::t) == 16, "what 16-byte aligned rows hold");

// Eight elements at p; wide: p is 16-byte aligned.
template <bool WIDE, class E>
DEV f8 load8(const E* p) {
    if constexpr (WIDE) {
        return __builtin_convertvector(*reinterpret_cast<const typename Vec8<E>::t*>(p), f8);
    } else {
        f8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
        return v;
    }
}

// Rounded to the nearest, ties to even.
template <bool WIDE, class E>
DEV void store8(E* p, f8 v) {
    if constexpr (WIDE) {
        *reinterpret_cast<typename Vec8<E>::t*>(p) = __builtin_convertvector(v, typename Vec8<E>::t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (E)v[i];
    }
}

// Cosine and sine of pair i at a position (row NULL: the position is outside
// the table, and the pair becomes NaN). NP pairs from an even i of a 16-byte
// aligned row, or one by one.
template <int NP, bool WIDE>
DEV void load_cs(const float* row, int i, float (&c)[NP], float (&s)[NP]) {
    const float nan = __builtin_nanf("");
    if constexpr (WIDE) {
        float4 v[NP / 2];
#pragma unroll
        for (int j = 0; j < NP / 2; ++j) v[j] = float4{nan, nan, nan, nan};
        if (row) {
#pragma unroll
            for (int j = 0; j < NP / 2; ++j) v[j] = *reinterpret_cast<const float4*>(row + 2 * (i + 2 * j));
        }
#pragma unroll
        for (int j = 0; j < NP; j += 2) c[j] = v[j / 2].x, s[j] = v[j / 2].y, c[j + 1] = v[j / 2].z, s[j + 1] = v[j / 2].w;
    } else {
#pragma unroll
        for (int j = 0; j < NP; ++j) c[j] = row ? row[2 * (i + j)] : nan, s[j] = row ? row[2 * (i + j) + 1] : nan;
    }
}

// The two halves of a rotation, each product and the sum rounded once.
DEV float turn_a(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    return a * c - b * s;
}
DEV float turn_b(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    return b * c + a * s;
}

}  // namespace gvr_elem

#endif  // GVR_ELEM_OPS_H
