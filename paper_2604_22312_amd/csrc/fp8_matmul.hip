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

// --- tiles through LDS
//
// A workgroup multiplies BM rows of A with BN rows of B, 128 elements at a time;
// the codes of a step come by direct loads into one of STAGES buffers in LDS while
// the steps before are multiplied. A row of a buffer is its 128 bytes in chunks of
// 16; chunk c of row r is at place c ^ (r & 7), so that eight lanes that read the
// same chunk of eight rows touch all banks once (the direct load's lanes write
// consecutive places, so it is their global addresses that are permuted). Lane l
// reads chunks l / 16 and l / 16 + 4 of its row: in both operands, so the sums are
// the same. Scales come four blocks at a time, four blocks ahead (a row's scales
// lie side by side: one block at a time would fetch each line four times).
//
// The direct loads are inline assembly, with no register result: the compiler
// would wait for all of them before every read of LDS, not knowing which buffer
// they write. drain<N>() waits until at most the newest N of them are under way,
// and for every LDS read of the wave, ahead of the barrier after which buffers
// change hands.
typedef unsigned v4u __attribute__((ext_vector_type(4)));

DEV v4u resource(const void* base, uint32_t bytes) {
    const uint64_t p = (uint64_t)(uintptr_t)base;
    return v4u{(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, bytes, 0x00020000u};
}
DEV uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
DEV v4u uniform(v4u v) { return v4u{uniform(v[0]), uniform(v[1]), uniform(v[2]), uniform(v[3])}; }

DEV void fetch16(uint32_t lds, v4u rsrc, uint32_t voffset, uint32_t soffset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "memory");
}
DEV void fetch4(uint32_t lds, v4u rsrc, uint32_t voffset, uint32_t soffset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "memory");
}
template <int N>
DEV void drain() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

template <int BM, int BN, int WM, int WN, int STAGES>
struct Tile {
    static constexpr int kWavesM = BM / WM, kWavesN = BN / WN, kWaves = kWavesM * kWavesN, kThreads = 64 * kWaves;
    static constexpr int kRows = BM + BN;
    static constexpr int kStage = kRows * kGroup;             // bytes of a step's codes
    static constexpr int kLoads = kStage / 1024 / kWaves;     // of a wave and step
    static constexpr int kSets = kRows / 64;                  // of 64 rows, whose scales a wave fetches at once
    static constexpr int kScales = 2 * 4 * kRows * 4;         // bytes: two windows of four blocks
    static constexpr int kLds = STAGES * kStage + kScales;
    static_assert(kStage % (1024 * kWaves) == 0 && BM % 64 == 0 && BN % 64 == 0 && kSets <= 2 * kWaves, "");
};

struct TileParams {
    MatmulParams p;
    float* parts;            // [splits][M][N] partial sums, or NULL: the results themselves
    uint32_t tiles_m, splits, steps, steps_each;   // blocks of 128 in all, and of a split
    uint32_t band;           // tiles of A that neighbouring workgroups share out before they move along B
};

template <class E, bool BYROW, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__((Tile<BM, BN, WM, WN, STAGES>::kThreads)) void tile_kernel(TileParams t) {
    using T = Tile<BM, BN, WM, WN, STAGES>;
    constexpr bool WIDE = sizeof(E) == 4;   // (sums on the float16 matrix cores)
    constexpr int NI = WN / 16, NJ = WM / 16;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    const MatmulParams& p = t.p;
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;

    // workgroups of one XCD (blockIdx.x % 8) take neighbouring tiles; those go down a band of A's tiles, then along B
    const uint32_t tiles = t.tiles_m * p.tiles_n, units = tiles * t.splits;
    uint32_t u = blockIdx.x;
    {
        const uint32_t xcd = u & 7, at = u >> 3, each = units >> 3, more = units & 7;
        u = xcd * each + min(xcd, more) + at;
    }
    const uint32_t split = uniform(u / tiles);   // (quotients are made in vector registers)
    u -= split * tiles;
    const uint32_t per_band = t.band * p.tiles_n, band = uniform(u / per_band), in = u - band * per_band;
    const uint32_t high = min(t.band, t.tiles_m - band * t.band), along = uniform(in / high);
    const int64_t m0 = (int64_t)(band * t.band + in - along * high) * BM, n0 = (int64_t)along * BN;
    const uint32_t first = split * t.steps_each, last = min(first + t.steps_each, t.steps);
    const uint32_t whole = (uint32_t)(p.K / kGroup);                 // steps of 128 elements; at most one more is shorter
    const uint32_t full = min(last, whole), n = full > first ? full - first : 0;

    // rows past the end read the last one and are not stored
    const int64_t left_m = min(p.M - m0, (int64_t)BM) - 1, left_n = min(p.N - n0, (int64_t)BN) - 1;
    const v4u ra = uniform(resource(p.a.codes + m0 * p.a.row_stride, 0xFFFFFFFFu));
    const v4u rb = uniform(resource(p.b.codes + n0 * p.b.row_stride, 0xFFFFFFFFu));
    const int64_t nb0 = n0 / p.b.rows_per_scale;
    const v4u rsa = uniform(resource(p.a.scale + m0 * p.a.scale_row_stride, 0xFFFFFFFFu));
    const v4u rsb = uniform(resource(p.b.scale + nb0 * p.b.scale_row_stride, 0xFFFFFFFFu));
    const uint32_t base = uniform((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds);
    uint32_t off[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int row = (wave * T::kLoads + i) * 8 + (lane >> 3);
        const uint32_t chunk = (lane & 7) ^ (row & 7);
        off[i] = row < BM ? (uint32_t)(min((int64_t)row, left_m) * p.a.row_stride) + 16 * chunk
                          : (uint32_t)(min((int64_t)(row - BM), left_n) * p.b.row_stride) + 16 * chunk;
    }
    constexpr int kMine = (T::kSets + T::kWaves - 1) / T::kWaves;    // sets of scales of a wave
    uint32_t scale_off[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int row = (wave + i * T::kWaves) * 64 + lane;
        scale_off[i] = row < BM ? (uint32_t)(min((int64_t)row, left_m) * p.a.scale_row_stride) * 4
                                : (uint32_t)(((n0 + min((int64_t)(row - BM), left_n)) / p.b.rows_per_scale - nb0) *
                                             p.b.scale_row_stride) * 4;
    }
    auto fetch_step = [&](uint32_t s) {   // s: of this workgroup's steps
        const uint32_t to = base + s % STAGES * T::kStage + wave * T::kLoads * 1024, at = (first + s) * kGroup;
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            const bool of_a = (wave * T::kLoads + i) * 8 < BM;   // (uniform: a load's eight rows are of one side)
            fetch16(to + i * 1024, of_a ? ra : rb, off[i], at);
        }
    };
    auto fetch_scales = [&](uint32_t s) {   // of steps s .. s + 3, s a multiple of 4
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int set = wave + i * T::kWaves;
            if (set < T::kSets) {
                const bool of_a = set * 64 < BM;
                const uint32_t to = base + STAGES * T::kStage + ((s >> 2 & 1) * 4 * T::kRows + set * 64) * 4;
                const uint32_t stride = (uint32_t)(of_a ? p.a.scale_block_stride : p.b.scale_block_stride) * 4;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (s + k < n) fetch4(to + k * T::kRows * 4, of_a ? rsa : rsb, scale_off[i], (first + s + k) * stride);
            }
        }
    };

    const int wm = wave % T::kWavesM * WM, wn = wave / T::kWavesM * WN;
    v4f acc[NI][NJ] = {};
    auto scaled = [&](int i, int j, v4f d, float sa, v4f sb) {
        if constexpr (BYROW) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * (sa * sb[r]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * sa;   // (sa holds both)
        }
    };
    if (n) {
        fetch_scales(0);
#pragma unroll
        for (uint32_t s = 0; s < STAGES - 1; ++s)
            if (s < n) fetch_step(s);
    }
    for (uint32_t s = 0; s < n; ++s) {
        // step s is in LDS when the newest STAGES - 2 steps' loads may be left
        if (s + STAGES - 1 <= n) drain<(STAGES - 2) * T::kLoads>();
        else drain<0>();
        if ((s & 3) == 0 && s + 4 < n) fetch_scales(s + 4);
        if (s + STAGES - 1 < n) fetch_step(s + STAGES - 1);
        const uint8_t* const codes = lds + s % STAGES * T::kStage;
        const float* const scales = reinterpret_cast<const float*>(lds + STAGES * T::kStage) + ((s >> 2 & 1) * 4 + (s & 3)) * T::kRows;
        auto fragment = [&](int row) {
            const uint8_t* const r = codes + row * kGroup;
            const v4u lo = *reinterpret_cast<const v4u*>(r + 16 * (quarter ^ (row & 7)));
            const v4u hi = *reinterpret_cast<const v4u*>(r + 16 * ((quarter + 4) ^ (row & 7)));
            return v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
        };
        v8i b[NI];
        v4f sb[NI];
        float sb1 = 1.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            b[i] = fragment(BM + wn + 16 * i + col);
            if constexpr (BYROW) sb[i] = *reinterpret_cast<const v4f*>(scales + BM + wn + 16 * i + 4 * quarter);
            else sb[i] = v4f{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (!BYROW) sb1 = scales[BM + wn];   // (WN rows of B from a multiple of WN share their scale)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const v8i a = fragment(wm + 16 * j + col);
            const float sa = scales[wm + 16 * j + col] * sb1;
            v4f d[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) d[i] = dot128<WIDE>(b[i], a);
#pragma unroll
            for (int i = 0; i < NI; ++i) scaled(i, j, d[i], sa, sb[i]);
        }
    }
    if (last > whole) {   // the last elements, less than 128
        const int64_t k = (int64_t)whole * kGroup + 32 * quarter;
        v8i b[NI];
        v4f sb[NI];
        const float* const scale = p.b.scale + whole * p.b.scale_block_stride;
        float sb1 = 1.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            b[i] = load32(p.b.codes + (n0 + min((int64_t)(wn + 16 * i + col), left_n)) * p.b.row_stride, k, p.K);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                sb[i][r] = BYROW ? scale[(n0 + min((int64_t)(wn + 16 * i + 4 * quarter + r), left_n)) * p.b.scale_row_stride] : 0.f;
        }
        if constexpr (!BYROW) sb1 = scale[(n0 + min((int64_t)wn, left_n)) / kGroup * p.b.scale_row_stride];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int64_t m = m0 + min((int64_t)(wm + 16 * j + col), left_m);
            const v8i a = load32(p.a.codes + m * p.a.row_stride, k, p.K);
            const float sa = p.a.scale[m * p.a.scale_row_stride + whole * p.a.scale_block_stride] * sb1;
#pragma unroll
            for (int i = 0; i < NI; ++i) scaled(i, j, dot128<WIDE>(b[i], a), sa, sb[i]);
        }
    }
    // four consecutive results of a row each
    const bool quads = (p.out_stride & 3) == 0 && ((uintptr_t)p.out & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int64_t m = m0 + wm + 16 * j + col;
        if (m >= p.M) continue;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t c = n0 + wn + 16 * i + 4 * quarter;
            if (t.parts) {
                float* const to = t.parts + ((int64_t)split * p.M + m) * p.N + c;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (c + r < p.N) to[r] = acc[i][j][r];
            } else {
                E* const to = static_cast<E*>(p.out) + m * p.out_stride + c;
                typedef E e4 __attribute__((ext_vector_type(4)));
                if (quads && c + 3 < p.N) {
                    *reinterpret_cast<e4*>(to) = __builtin_convertvector(acc[i][j], e4);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c + r < p.N) to[r] = (E)acc[i][j][r];
                }
            }
        }
    }
}

// Sums of the splits' parts, in their order.
template <class E>
__global__ __launch_bounds__(gvr_fp8::kThreads) void join_kernel(TileParams t) {
    const MatmulParams& p = t.p;
    const int64_t at = (int64_t)blockIdx.x * gvr_fp8::kThreads + threadIdx.x, total = p.M * p.N;
    if (at >= total) return;
    float sum = 0.f;
    for (uint32_t s = 0; s < t.splits; ++s) sum += t.parts[s * total + at];
    const int64_t m = at / p.N, n = at - m * p.N;
    static_cast<E*>(p.out)[m * p.out_stride + n] = (E)sum;
}

template <class E>
gvr_status launch(const TileParams& t, const gvr_fp8::MatmulPlan& plan, void* stream) {
    const dim3 grid((unsigned)plan.workgroups);
    const hipStream_t s = (hipStream_t)stream;
    const bool by_row = t.p.b.rows_per_scale == 1;
    switch (plan.shape) {
        case gvr_fp8::kAnyShape:
            hipLaunchKernelGGL(matmul_kernel<E>, grid, dim3(gvr_fp8::kThreads), 0, s, t.p);
            break;
        case gvr_fp8::kLarge:
            if constexpr (sizeof(E) == 2) {
                if (by_row) hipLaunchKernelGGL((tile_kernel<E, true, 256, 256, 128, 64, 2>), grid, dim3(512), 0, s, t);
                else hipLaunchKernelGGL((tile_kernel<E, false, 256, 256, 128, 64, 2>), grid, dim3(512), 0, s, t);
            }
            break;
        default:
            if (by_row) hipLaunchKernelGGL((tile_kernel<E, true, 128, 128, 64, 64, 2>), grid, dim3(256), 0, s, t);
            else hipLaunchKernelGGL((tile_kernel<E, false, 128, 128, 64, 64, 2>), grid, dim3(256), 0, s, t);
    }
    if (t.parts)
        hipLaunchKernelGGL(join_kernel<E>, dim3((unsigned)((t.p.M * t.p.N + gvr_fp8::kThreads - 1) / gvr_fp8::kThreads)),
                           dim3(gvr_fp8::kThreads), 0, s, t);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // namespace

extern "C" {

gvr_status gvr_fp8_matmul_workspace(const gvr_fp8_matrix* a, const gvr_fp8_matrix* b, int64_t M, int64_t N, int64_t K,
                                    size_t* bytes) {
    if (!bytes) return GVR_ERR_INVALID_ARG;
    *bytes = 0;
    const gvr_status st = gvr_fp8::check_matmul(a, b, M, N, K, false);
    if (st != GVR_OK || M == 0 || N == 0) return st;
    gvr_fp8::MatmulPlan plan;
    const gvr_status fits = gvr_fp8::plan_matmul(*a, *b, M, N, K, false, (size_t)-1, &plan);
    if (fits == GVR_OK) *bytes = plan.workspace;
    return fits;
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
    const gvr_status fits = gvr_fp8::plan_matmul(*a, *b, M, N, K, size == 4, ws_bytes, &plan);
    if (fits != GVR_OK) return fits;
    TileParams t;
    t.p.a = *a, t.p.b = *b, t.p.out = out;
    t.p.M = M, t.p.N = N, t.p.K = K, t.p.out_stride = out_stride;
    t.p.tiles_n = (uint32_t)plan.tiles_n;
    t.parts = plan.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    t.tiles_m = (uint32_t)plan.tiles_m;
    t.splits = (uint32_t)plan.splits;
    t.steps = (uint32_t)gvr_fp8::groups_of(K);
    t.steps_each = (uint32_t)plan.steps_each;
    t.band = (uint32_t)plan.band;
    return dtype == GVR_BF16 ? launch<__bf16>(t, plan, stream)
           : dtype == GVR_F16 ? launch<_Float16>(t, plan, stream) : launch<float>(t, plan, stream);
}

}  // extern "C"
