// fp8_matmul.hip -- products of 8-bit matrices with a scale per 128 elements,
// behind include/gvr_fp8.h.
//
// A wave multiplies 16 rows of B with 64 rows of A, 128 elements at a time: one
// gfx950 v_mfma_f32_16x16x128_f8f6f4 per 16 x 16 results gives the sum of a whole
// block, which is scaled and added in float32. Lane l holds, of row l % 16 of
// both operands, the 32 bytes from 32 (l / 16) on, and of the results column
// l % 16 (a row of A) and rows 4 (l / 16) + i (of B).
//
// The FP8 matrix cores add the products of eight consecutive elements in fixed
// point: measured, a product below 2^-13 of the largest of its eight is lost (with
// one of 2^16 in a group, 2^3 counts and 2^2 does not), between groups float32 is
// kept. On normal codes that is 2^-19 of the sum of the magnitudes, a hundredth of a
// bfloat16 result's rounding, but 30 times a float32 sum's. Results in float32 are
// therefore summed by the float16 matrix cores, which hold every code and add in
// float32 (2^-30 of the magnitudes for 32 products), at half the rate.

#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

#include "gvr_fp8.h"
#include "fp8_plan.h"

#ifndef DEV
#define DEV __device__ __forceinline__
#endif

namespace {

using gvr_fp8::kGroup;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

struct MatmulParams {
    gvr_fp8_matrix a, b;
    void* out;
    int64_t M, N, K, out_stride;
    uint32_t tiles_n;
};

// Bytes k .. k+31 of a row of K, zeros past its end; any alignment.
DEV v8i load32(const uint8_t* row, int64_t k, int64_t K) {
    v8i v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k + 32 <= K) {
        memcpy(&v, row + k, 32);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + 4 * i + j < K) w |= (uint32_t)row[k + 4 * i + j] << (8 * j);
            v[i] = (int)w;
        }
    }
    return v;
}

// Eight codes as float16.
DEV h8 widen(int lo, int hi) {
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A block's sums; WIDE: on the float16 matrix cores.
template <bool WIDE>
DEV v4f dot128(v8i a, v8i b) {
    v4f d = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(a[i], a[i + 1]), widen(b[i], b[i + 1]), d, 0, 0, 0);
        return d;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, d, 0, 0, 0, 0, 0, 0);
    }
}

template <class E>
__global__ __launch_bounds__(gvr_fp8::kThreads) void matmul_kernel(MatmulParams p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const int64_t m0 = (int64_t)(blockIdx.x / p.tiles_n) * gvr_fp8::kTileM;
    const int64_t n0 = (int64_t)(blockIdx.x % p.tiles_n) * gvr_fp8::kTileN + 16 * wave;
    if (n0 >= p.N) return;
    // rows past the end read the last one and are not stored
    const int64_t nb = min(n0 + col, p.N - 1);
    const uint8_t* const b = p.b.codes + nb * p.b.row_stride;
    const uint8_t* a[4];
    const float* sa[4];
    const float* sb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t m = min(m0 + 16 * j + col, p.M - 1);
        a[j] = p.a.codes + m * p.a.row_stride;
        sa[j] = p.a.scale + m * p.a.scale_row_stride;
        sb[j] = p.b.scale + min(n0 + 4 * quarter + j, p.N - 1) / p.b.rows_per_scale * p.b.scale_row_stride;
    }
    v4f acc[4] = {};
    for (int64_t k = 0, g = 0; k < p.K; k += kGroup, ++g) {
        const v8i bv = load32(b, k + 32 * quarter, p.K);
        float s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = sb[i][g * p.b.scale_block_stride];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v4f d = dot128<sizeof(E) == 4>(bv, load32(a[j], k + 32 * quarter, p.K));
            const float t = sa[j][g * p.a.scale_block_stride];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] += d[i] * (t * s[i]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t m = m0 + 16 * j + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t n = n0 + 4 * quarter + i;
            if (m < p.M && n < p.N) static_cast<E*>(p.out)[m * p.out_stride + n] = (E)acc[j][i];
        }
    }
}

template <class E>
gvr_status launch(const MatmulParams& p, unsigned workgroups, void* stream) {
    hipLaunchKernelGGL(matmul_kernel<E>, dim3(workgroups), dim3(gvr_fp8::kThreads), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // namespace

extern "C" {

gvr_status gvr_fp8_matmul_workspace(const gvr_fp8_matrix* a, const gvr_fp8_matrix* b, int64_t M, int64_t N, int64_t K,
                                    size_t* bytes) {
    if (!bytes) return GVR_ERR_INVALID_ARG;
    *bytes = 0;
    return gvr_fp8::check_matmul(a, b, M, N, K, false);
}

gvr_status gvr_fp8_matmul(const gvr_fp8_matrix* a, const gvr_fp8_matrix* b, int64_t M, int64_t N, int64_t K, void* out,
                          int64_t out_stride, int32_t dtype, void* workspace, size_t ws_bytes, void* stream) {
    const gvr_status st = gvr_fp8::check_matmul(a, b, M, N, K, true);
    if (st != GVR_OK) return st;
    const int size = gvr_rot::dtype_size(dtype);
    if (size == 0 || ((uintptr_t)out & (size - 1)) || ((uintptr_t)workspace & 15) || (!workspace && ws_bytes))
        return GVR_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return GVR_OK;
    if (!out) return GVR_ERR_INVALID_ARG;
    gvr_fp8::MatmulPlan plan;
    const gvr_status fits = gvr_fp8::plan_matmul(M, N, &plan);
    if (fits != GVR_OK) return fits;
    MatmulParams p;
    p.a = *a, p.b = *b, p.out = out;
    p.M = M, p.N = N, p.K = K, p.out_stride = out_stride;
    p.tiles_n = (uint32_t)plan.tiles_n;
    const unsigned n = (unsigned)plan.workgroups;
    return dtype == GVR_BF16 ? launch<__bf16>(p, n, stream)
           : dtype == GVR_F16 ? launch<_Float16>(p, n, stream) : launch<float>(p, n, stream);
}

}  // extern "C"
