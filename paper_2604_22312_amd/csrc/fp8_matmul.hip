// fp8_matmul.hip -- products of 8-bit matrices with a scale per 128 elements,
// behind include/gvr_fp8.h.
//
// One gfx950 v_mfma_f32_16x16x128_f8f6f4 multiplies 16 rows of B with 16 rows of A over
// 128 elements and so gives the sums of a whole block, which are scaled and added in
// float32: four multiply-adds of 4 cycles to a matrix instruction of 32. Lane l holds 32
// bytes of row l % 16 of both operands, and of the results column l % 16 (a row of A)
// and rows 4 (l / 16) + i (of B), so that a lane's results share A's scale and lie
// together in memory.
//
// Three kinds of kernels, chosen by sizes and alignment in fp8_plan.h: few rows of A
// (codes from memory to registers), tiles through LDS, and one for rows that are not
// 16-byte aligned where the workspace has no room for copies: it loads pieces of any
// alignment and shares nothing (128 x 4096 x 4099 in packed rows 115 us, copied first 25, in
// rows of 4112 bytes 16.7).
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
//
// 8192 x 8192 x 4096 into bfloat16 takes 243 to 251 us = 2.2 PFLOP/s (256 x 256 tiles; 183 us =
// 3.0 PFLOP/s is a library product of the same codes with one scale for all). The card
// runs at 1.9 GHz then, where the matrix instructions alone take 139 us. Measured in copies
// that leave parts out: without fetching codes 20 us less, without the stores of the
// results 22 us less (a compute unit stores its 128 KB in 5 us and multiplies
// nothing meanwhile; its LDS holds one workgroup), the rest is waves waiting for each
// other at the barrier. The steps that led here: additions in the shadow of the matrix
// instructions (270 -> 260), the last tiles behind the barrier with loads spread out
// (290 -> 275), results in 16-byte stores (252 -> 234).
// Smaller products are bound by a compute unit's intake, some 30 to 60 GB/s, and by the
// steps' latency: 128 x 8192 x 4096 17.5 us, of which joining two splits 4.
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

DEV v4u resource(const void* base, uint32_t bytes) {
    const uint64_t p = (uint64_t)(uintptr_t)base;
    return v4u{(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, bytes, 0x00020000u};
}
DEV uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
DEV v4u uniform(v4u v) { return v4u{uniform(v[0]), uniform(v[1]), uniform(v[2]), uniform(v[3])}; }

// (both say that they write m0: the compiler keeps numbers of its own there for other instructions. That it warns of naming
// a register that it hands out by itself is about asm that expects to find its own number there afterwards)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
DEV void fetch16(uint32_t lds, v4u rsrc, uint32_t voffset, uint32_t soffset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "m0", "memory");
}
DEV void fetch4(uint32_t lds, v4u rsrc, uint32_t voffset, uint32_t soffset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "m0", "memory");
}
#pragma clang diagnostic pop
template <int N>
DEV void drain() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

template <int V>
struct Int {
    constexpr operator int() const { return V; }
};
template <int N, int I = 0, class F>
DEV void each(F& f) {   // f(0) .. f(N - 1), known when compiled
    if constexpr (I < N) {
        f(Int<I>());
        each<N, I + 1>(f);
    }
}

template <int BM, int BN, int WM, int WN, int STAGES>
struct Tile {
    static constexpr int kWavesM = BM / WM, kWavesN = BN / WN, kWaves = kWavesM * kWavesN, kThreads = 64 * kWaves;
    static constexpr int kRows = BM + BN;
    static constexpr int kStage = kRows * kGroup;             // bytes of a step's codes
    static constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves, kLoads = kLoadsA + kLoadsB;   // of a wave and step
    static constexpr int kSets = kRows / 64;                  // of 64 rows, whose scales a wave fetches at once
    static constexpr int kScales = 2 * 4 * kRows * 4;         // bytes: two windows of four blocks
    static constexpr int kLds = STAGES * kStage + kScales;
    static_assert(STAGES <= 5, "scales come four steps ahead");
    static_assert(WM % 32 == 0 && WN % 32 == 0, "tiles go in pairs");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && BM % 64 == 0 && BN % 64 == 0 && kLoads <= 8, "");
};

struct TileParams {
    MatmulParams p;
    float* parts;            // [splits][M][N] partial sums, or NULL: the results themselves
    uint32_t tiles_m, splits, steps, steps_each;   // blocks of 128 in all, and of a split
    uint32_t join_cols;      // workgroups of a row of results in the kernel that adds the parts
    bool quads;              // four scales of a row lie together, 16-byte aligned, in both matrices
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
    const uint32_t n = last > first ? last - first : 0;

    // rows past the end read the last one and are not stored
    const int64_t left_m = min(p.M - m0, (int64_t)BM) - 1, left_n = min(p.N - n0, (int64_t)BN) - 1;
    const int64_t nb0 = n0 / p.b.rows_per_scale;
    v4u ra = uniform(resource(p.a.codes + m0 * p.a.row_stride, 0xFFFFFFFFu));
    v4u rb = uniform(resource(p.b.codes + n0 * p.b.row_stride, 0xFFFFFFFFu));
    v4u rsa = uniform(resource(p.a.scale + m0 * p.a.scale_row_stride, 0xFFFFFFFFu));
    v4u rsb = uniform(resource(p.b.scale + nb0 * p.b.scale_row_stride, 0xFFFFFFFFu));
    // (a scalar register that a vector instruction has written may be read by a load five states later; the compiler does not
    // count them for loads in assembly)
    asm volatile("s_nop 4" : "+s"(ra), "+s"(rb), "+s"(rsa), "+s"(rsb));
    const uint32_t base = uniform((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds);
    // A wave's loads are of eight consecutive rows each, first kLoadsA of A's, then of B's: the first ones' offsets, and the last rows'.
    const uint32_t chunk = 16 * ((lane & 7) ^ (lane >> 3)), a_stride = (uint32_t)p.a.row_stride, b_stride = (uint32_t)p.b.row_stride;
    uint32_t off_a = (wave * T::kLoadsA * 8 + (lane >> 3)) * a_stride + chunk, off_b = (wave * T::kLoadsB * 8 + (lane >> 3)) * b_stride + chunk;
    const uint32_t last_a = (uint32_t)left_m * a_stride + chunk, last_b = (uint32_t)left_n * b_stride + chunk;
    auto load_offset = [&](int i) {
        return i < T::kLoadsA ? min(off_a + i * 8 * a_stride, last_a) : min(off_b + (i - T::kLoadsA) * 8 * b_stride, last_b);
    };
    auto load_place = [&](int i) {   // in a buffer
        return (uint32_t)(i < T::kLoadsA ? wave * T::kLoadsA + i : BM / 8 + wave * T::kLoadsB + i - T::kLoadsA) * 1024;
    };
    constexpr int kMine = (T::kSets + T::kWaves - 1) / T::kWaves;    // sets of scales of a wave
    uint32_t scale_off[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int row = (wave + i * T::kWaves) * 64 + lane;
        scale_off[i] = row < BM ? (uint32_t)(min((int64_t)row, left_m) * p.a.scale_row_stride) * 4
                                : (uint32_t)(((n0 + min((int64_t)(row - BM), left_n)) / p.b.rows_per_scale - nb0) *
                                             p.b.scale_row_stride) * 4;
    }
    // bytes from a row's scale to the next row's and the next block's, in LDS
    const uint32_t by_row = t.quads ? 16 : 4, by_block = t.quads ? 4 : 4 * T::kRows;
    // Loads FROM .. TO - 1 of a step (s: of this workgroup's steps).
    auto fetch_codes = [&](uint32_t s, auto FROM, auto TO) {
        const uint32_t lds_to = base + s % STAGES * T::kStage, at = (first + s) * kGroup;
        asm volatile("" : "+v"(off_a), "+v"(off_b));   // (the offsets are made anew each time, not held in registers)
#pragma unroll
        for (int i = FROM; i < TO; ++i) fetch16(lds_to + load_place(i), i < T::kLoadsA ? ra : rb, load_offset(i), at);
    };
    // The last elements, less than 128, and zeros behind them: whole chunks first, then the one that ends inside (a lane a row).
    auto copy_rest = [&](uint32_t s) {
        const uint32_t lds_to = base + s % STAGES * T::kStage, at = (first + s) * kGroup;
        const uint8_t *const codes_a = p.a.codes + m0 * p.a.row_stride + at, *const codes_b = p.b.codes + n0 * p.b.row_stride + at;
        const int left = (int)(p.K - at), mine = left - (int)chunk;
        v4u v[T::kLoads];
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            v[i] = v4u{0, 0, 0, 0};
            if (mine >= 16) v[i] = *reinterpret_cast<const v4u*>((i < T::kLoadsA ? codes_a : codes_b) + load_offset(i));
        }
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) *(__attribute__((address_space(3))) v4u*)(uintptr_t)(lds_to + load_place(i) + lane * 16) = v[i];
        if ((left & 15) && lane < 8 * T::kLoads) {
            const bool of_a = lane < 8 * T::kLoadsA;
            const int row = of_a ? wave * T::kLoadsA * 8 + lane : wave * T::kLoadsB * 8 + lane - 8 * T::kLoadsA;
            const uint8_t* const from = (of_a ? codes_a + min((int64_t)row, left_m) * a_stride
                                              : codes_b + min((int64_t)row, left_n) * b_stride) + (left & ~15);
            v4u w = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 15; ++k)
                if (k < (left & 15)) w[k / 4] |= (uint32_t)from[k] << (8 * (k & 3));
            *(__attribute__((address_space(3))) v4u*)(uintptr_t)(lds_to + (of_a ? row : BM + row) * 128 + 16 * ((left >> 4) ^ (row & 7))) = w;
        }
    };
    auto fetch_scales = [&](uint32_t s) {   // of steps s .. s + 3, s a multiple of 4
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int set = wave + i * T::kWaves;
            if (set < T::kSets) {
                const bool of_a = set * 64 < BM;
                const uint32_t to = base + STAGES * T::kStage + (s >> 2 & 1) * 16 * T::kRows + set * 64 * by_row;
                if (t.quads) {
                    fetch16(to, of_a ? rsa : rsb, scale_off[i], (first + s) * 4);
                } else {
                    const uint32_t stride = (uint32_t)(of_a ? p.a.scale_block_stride : p.b.scale_block_stride) * 4;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (s + k < n) fetch4(to + k * by_block, of_a ? rsa : rsb, scale_off[i], (first + s + k) * stride);
                }
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
    // Addresses of this lane's codes in the first tile of its wave, of either side: chunk l / 16 of its row, and chunk l / 16 + 4
    // 64 bytes before or behind. Tiles are 2048 bytes apart, steps kStage.
    typedef const __attribute__((address_space(3))) v4u* Chunk;
    typedef const __attribute__((address_space(3))) float* Number;
    const uint32_t in_tile = col * kGroup + 16 * (quarter ^ (col & 7));
    const uint32_t a_at = base + wm * kGroup + in_tile, b_at = base + (BM + wn) * kGroup + in_tile;
    auto fragment = [&](uint32_t at, int tile) {
        const v4u lo = *(Chunk)(uintptr_t)(at + tile * 2048), hi = *(Chunk)(uintptr_t)((at ^ 64) + tile * 2048);
        return v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    v8i b[NI], a[2];
    v4f sb[NI] = {};
    float sb1 = 1.f;
    auto stage = [&](uint32_t s) { return s % STAGES * T::kStage; };
    // A step's loads are spread over the tiles of A that follow the barrier which frees their buffer (the last two of a step and
    // the first of the next), so that no wave is held up by a full queue of them: kIssued[x] of them after x of these tiles.
    constexpr int kSlots = 4;
    constexpr auto issued = [](int x) { return x >= kSlots ? T::kLoads : (x * T::kLoads + kSlots - 1) / kSlots; };
    constexpr int kHead = issued(2);   // loads ahead of a step's end
    const uint32_t loaded = min(last, whole) > first ? min(last, whole) - first : 0;   // steps that direct loads bring
    auto load_sb = [&](uint32_t window) {
        if constexpr (BYROW)
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sb[i][r] = *(Number)(uintptr_t)(window + (BM + wn + 16 * i + 4 * quarter + r) * by_row);
    };
    v4f d[2][NI] = {};
    float f_before = 0.f;
    // LEFT: the loads of step s - 1 + STAGES that the step before left; HEAD: the first of step s + STAGES.
    auto step = [&](uint32_t s, auto LEFT, auto HEAD) {
        if ((s & 3) == 0 && s + 4 < n) fetch_scales(s + 4);
        const uint32_t window = base + STAGES * T::kStage + (s >> 2 & 1) * 16 * T::kRows + (s & 3) * by_block;
        uint32_t sa_at = window + (wm + col) * by_row;
        if constexpr (!BYROW) sb1 = *(Number)(uintptr_t)(window + (BM + wn) * by_row);   // (WN rows of B from a multiple of WN share it)
        const uint32_t a_now = a_at + stage(s), a_then = a_at + stage(s + 1), b_then = b_at + stage(s + 1);
        auto next_sa = [&] {
            const float v = *(Number)(uintptr_t)sa_at;
            sa_at += 16 * by_row;
            asm volatile("" : "+v"(sa_at));   // (one running address)
            return v;
        };
        float sa = next_sa(), sa_next = next_sa();
        auto tile = [&](auto J) {
            constexpr int j = J;
            if constexpr (j == NJ - 2) {
                // The step's last two tiles are multiplied behind the barrier, from registers, while the next step's codes are
                // read: step s + 1 is in LDS when the newest STAGES - 2 steps' loads may be left, and this step's buffer is free.
                if constexpr (HEAD) drain<(STAGES - 2) * T::kLoads>();
                else drain<0>();
                if constexpr (LEFT && !HEAD)
                    if (n > loaded) copy_rest(loaded);   // (s + STAGES)
            }
            if constexpr (HEAD && j >= NJ - 2)
                fetch_codes(s + STAGES, Int<issued(j - NJ + 2)>(), Int<issued(j - NJ + 3)>());
            if constexpr (LEFT && j + 2 < kSlots)
                fetch_codes(s - 1 + STAGES, Int<issued(j + 2)>(), Int<issued(j + 3)>());
            // A tile's sums are scaled and added while the next one's are made, four additions to a matrix instruction: one wave's
            // vector instructions run in the shadow of its own matrix instructions.
            constexpr int before = (j + NJ - 1) % NJ;
            const float f = sa * sb1;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if (i == 0) __builtin_amdgcn_s_setprio(1);   // (the other wave of the unit is to read and add meanwhile)
                d[j & 1][i] = dot128<WIDE>(b[i], a[j & 1]);
                if (i == NI - 1) __builtin_amdgcn_s_setprio(0);
                if constexpr (j == NJ - 1) b[i] = fragment(b_then, i);   // (behind the last step: read and not used)
                if (i == NI - 1) a[j & 1] = j + 2 < NJ ? fragment(a_now, j + 2) : fragment(a_then, j + 2 - NJ);
                scaled(i, before, d[(j + 1) & 1][i], f_before, sb[i]);
                asm volatile("" : "+v"(acc[i][before]));   // (added here: moved behind the branches, sums and products would not fit the registers)
                __builtin_amdgcn_sched_barrier(0);
            }
            f_before = f;
            if constexpr (j == 0) load_sb(window);
            sa = sa_next;
            if constexpr (j + 2 < NJ) sa_next = next_sa();
        };
        each<NJ>(tile);
    };
    if (n) {
        fetch_scales(0);
        const bool ring = loaded >= STAGES;
#pragma unroll
        for (uint32_t s = 0; s < STAGES - 1; ++s)
            if (s < loaded) fetch_codes(s, Int<0>(), Int<T::kLoads>());
        if (ring) fetch_codes(STAGES - 1, Int<0>(), Int<kHead>());
        else if (n > loaded) copy_rest(loaded);
        if (ring) drain<(STAGES - 2) * T::kLoads + kHead>();
        else drain<0>();
#pragma unroll
        for (int i = 0; i < NI; ++i) b[i] = fragment(b_at, i);
        a[0] = fragment(a_at, 0);
        a[1] = fragment(a_at, 1);
        uint32_t s = 0;
        if (ring) {
            for (; s + STAGES < loaded; ++s) step(s, Int<1>(), Int<1>());
            step(s++, Int<1>(), Int<0>());
        }
        for (; s < n; ++s) step(s, Int<0>(), Int<0>());
#pragma unroll
        for (int i = 0; i < NI; ++i) scaled(i, NJ - 1, d[1][i], f_before, sb[i]);
    }
    // A lane holds four consecutive results of a row in each tile; of 16-bit results two neighbouring tiles exchange lanes, so
    // that it stores eight (8-byte stores cost the large product 18 us of 252).
    typedef E e4 __attribute__((ext_vector_type(4)));
    const bool rows16 = ((p.out_stride * (int)sizeof(E)) & 15) == 0 && ((uintptr_t)p.out & 15) == 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int64_t m = m0 + wm + 16 * j + col;
        if constexpr (sizeof(E) == 2) {
            // (whole rows of lanes take part in the exchange, also those past the end)
            if (!t.parts && rows16 && n0 + wn + WN <= p.N) {
#pragma unroll
                for (int i = 0; i < NI; i += 2) {
                    const v2u x = __builtin_bit_cast(v2u, __builtin_convertvector(acc[i][j], e4));
                    const v2u y = __builtin_bit_cast(v2u, __builtin_convertvector(acc[i + 1][j], e4));
                    v4u r;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const auto s = __builtin_amdgcn_permlane32_swap(x[k], y[k], false, false);
                        const auto q = __builtin_amdgcn_permlane16_swap(s[0], s[1], false, false);
                        r[k] = q[0], r[2 + k] = q[1];
                    }
                    if (m < p.M)
                        *reinterpret_cast<v4u*>(static_cast<E*>(p.out) + m * p.out_stride + n0 + wn + 16 * i + 8 * quarter) = r;
                }
                continue;
            }
        }
        if (m >= p.M) continue;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t c = n0 + wn + 16 * i + 4 * quarter;
            float* const part = t.parts ? t.parts + ((int64_t)split * p.M + m) * p.N + c : nullptr;
            E* const to = static_cast<E*>(p.out) + m * p.out_stride + c;
            if (part && (p.N & 3) == 0) {
                if (c < p.N) *reinterpret_cast<v4f*>(part) = acc[i][j];
            } else if (!part && sizeof(E) == 4 && rows16 && c + 3 < p.N) {
                *reinterpret_cast<e4*>(to) = __builtin_convertvector(acc[i][j], e4);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (c + r < p.N) {
                        if (part) part[r] = acc[i][j][r];
                        else to[r] = (E)acc[i][j][r];
                    }
            }
        }
    }
}

// --- up to 32 rows of A
//
// A workgroup multiplies 16 NT rows of B with all rows of A (at most 16 MT); its
// waves share out the blocks of 128 and their sums are added at the end, in the order
// of the waves. Codes go from memory to registers, AHEAD blocks of a wave at a time,
// with no barrier on the way; lanes whose row A does not have load nothing. Lane l
// holds chunks l / 16 and l / 16 + 4 of its rows.
// Bound by how fast a compute unit takes in B (1 x 8192 x 4096: 34 MB in 8.0 us =
// 4.2 TB/s; 1 x 4096 x 4096: 5.9, of which launch and sums 3.5) and A's rows beside it
// (16 rows: 9.7). Up to 16 rows the tile kernels take 11.7 us on 8192 rows of B, with
// 17 and 32 rows on 4096 of them 11.2 and 11.8 against 7.9 and 9.7; on 8192 the two
// are even at 32 rows (12.4, 12.6), with 64 rows the tiles are ahead (13.2).

// Chunks `quarter` and `quarter` + 4 of a row's 128 bytes; REST: of the last ones, zeros past `left`.
template <bool REST>
DEV v8i load_chunks(const uint8_t* row, int quarter, int left) {
    v4u v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = 64 * h + 16 * quarter;
        if (!REST || left >= at + 16) {
            v[h] = *reinterpret_cast<const v4u*>(row + at);
        } else {
            v[h] = v4u{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (at + i < left) v[h][i / 4] |= (uint32_t)row[at + i] << (8 * (i & 3));
        }
    }
    return v8i{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3], (int)v[1][0], (int)v[1][1], (int)v[1][2], (int)v[1][3]};
}

template <class E, bool BYROW, int MT, int NT, int AHEAD, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void rows_kernel(MatmulParams p) {
    constexpr bool WIDE = sizeof(E) == 4;
    __shared__ v4f sums[WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
    // rows of B past the end read the last one and are not stored, those of A are zeros
    const uint8_t* a[MT];
    const float* sa[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int m = 16 * j + col < p.M ? 16 * j + col : 0;
        a[j] = p.a.codes + m * p.a.row_stride;
        sa[j] = p.a.scale + m * p.a.scale_row_stride;
    }
    const uint8_t* b[NT];
    const float* sb[BYROW ? 4 * NT : 1];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        b[i] = p.b.codes + min(n0 + 16 * i + col, p.N - 1) * p.b.row_stride;
        if constexpr (BYROW)
#pragma unroll
            for (int r = 0; r < 4; ++r) sb[4 * i + r] = p.b.scale + min(n0 + 16 * i + 4 * quarter + r, p.N - 1) * p.b.scale_row_stride;
    }
    if constexpr (!BYROW) sb[0] = p.b.scale + min(n0, p.N - 1) / kGroup * p.b.scale_row_stride;   // (16 NT rows from a multiple of 16 NT share it)
    v4f acc[NT][MT] = {};
    auto add = [&](const v8i (&bv)[NT], const float (&fb)[BYROW ? 4 * NT : 1], const v8i (&av)[MT], const float (&fa)[MT]) {
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const v4f d = dot128<WIDE>(bv[i], av[j]);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * (fa[j] * fb[BYROW ? 4 * i + r : 0]);
            }
    };
    auto load = [&](int64_t s, auto REST, v8i (&bv)[NT], float (&fb)[BYROW ? 4 * NT : 1], v8i (&av)[MT], float (&fa)[MT]) {
        const int left = (int)min(p.K - s * kGroup, (int64_t)kGroup);
#pragma unroll
        for (int i = 0; i < NT; ++i) bv[i] = load_chunks<REST>(b[i] + s * kGroup, quarter, left);
#pragma unroll
        for (int i = 0; i < (BYROW ? 4 * NT : 1); ++i) fb[i] = sb[i][s * p.b.scale_block_stride];
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            av[j] = v8i{0, 0, 0, 0, 0, 0, 0, 0};
            fa[j] = 0.f;
            if (16 * j + col < p.M) {
                av[j] = load_chunks<REST>(a[j] + s * kGroup, quarter, left);
                fa[j] = sa[j][s * p.a.scale_block_stride];
            }
        }
    };
    const int64_t whole = p.K / kGroup;
    for (int64_t s0 = wave; s0 < whole; s0 += WAVES * AHEAD) {
        v8i bv[AHEAD][NT], av[AHEAD][MT];
        float fb[AHEAD][BYROW ? 4 * NT : 1], fa[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)   // (behind the end: the first block again, not added)
            load(s0 + u * WAVES < whole ? s0 + u * WAVES : s0, Int<0>(), bv[u], fb[u], av[u], fa[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s0 + u * WAVES < whole) add(bv[u], fb[u], av[u], fa[u]);
    }
    if (p.K > whole * kGroup && whole % WAVES == wave) {
        v8i bv[NT], av[MT];
        float fb[BYROW ? 4 * NT : 1], fa[MT];
        load(whole, Int<1>(), bv, fb, av, fa);
        add(bv, fb, av, fa);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < MT; ++j) sums[wave][j][lane] = acc[i][j];
        __syncthreads();
        for (int at = threadIdx.x; at < MT * 256; at += 64 * WAVES) {
            // rows of results first, so that a row's results lie together
            const int m = at / 16, c = at % 16, l = m % 16 + 16 * (c >> 2);
            const int64_t n = n0 + 16 * i + c;
            if (m < p.M && n < p.N) {
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) sum += sums[w][m >> 4][l][c & 3];
                static_cast<E*>(p.out)[m * p.out_stride + n] = (E)sum;
            }
        }
    }
}

// Sums of the splits' parts, in their order; a thread takes four results of a row, a workgroup 1024.
template <class E>
__global__ __launch_bounds__(gvr_fp8::kThreads) void join_kernel(TileParams t) {
    const MatmulParams& p = t.p;
    const int64_t m = blockIdx.x / t.join_cols, n = ((int64_t)(blockIdx.x % t.join_cols) * gvr_fp8::kThreads + threadIdx.x) * 4;
    if (n >= p.N) return;
    const int64_t total = p.M * p.N;
    const float* from = t.parts + m * p.N + n;
    E* const to = static_cast<E*>(p.out) + m * p.out_stride + n;
    v4f sum = {0.f, 0.f, 0.f, 0.f};
    if ((p.N & 3) == 0) {
        for (uint32_t s = 0; s < t.splits; ++s, from += total) sum += *reinterpret_cast<const v4f*>(from);
    } else {
        for (uint32_t s = 0; s < t.splits; ++s, from += total)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < p.N) sum[r] += from[r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n + r < p.N) to[r] = (E)sum[r];
}

// Rows of codes to rows that 16-byte loads can serve, a thread 16 bytes; A's, then B's.
struct CopyParams {
    const uint8_t* from[2];
    uint8_t* to[2];
    int64_t stride[2], to_stride, K;
    uint32_t items[2], chunks;   // of 16 bytes, in all and of a row
};
__global__ __launch_bounds__(gvr_fp8::kThreads) void copy_kernel(CopyParams p) {
    uint32_t i = blockIdx.x * (uint32_t)gvr_fp8::kThreads + threadIdx.x;
    const int side = i >= p.items[0];
    if (side) i -= p.items[0];
    if (i >= p.items[side]) return;
    const uint32_t r = i / p.chunks, c = i - r * p.chunks;
    const uint8_t* const from = p.from[side] + r * p.stride[side] + 16 * (int64_t)c;
    const int64_t left = p.K - 16 * (int64_t)c;
    v4u v = {0, 0, 0, 0};
    if (left >= 16) {
        memcpy(&v, from, 16);
    } else {
#pragma unroll
        for (int k = 0; k < 15; ++k)
            if (k < left) v[k / 4] |= (uint32_t)from[k] << (8 * (k & 3));
    }
    *reinterpret_cast<v4u*>(p.to[side] + r * p.to_stride + 16 * (int64_t)c) = v;
}

template <class E, bool BYROW>
void launch_shape(const TileParams& t, const gvr_fp8::MatmulPlan& plan, hipStream_t s) {
    const dim3 grid((unsigned)plan.workgroups), block(plan.threads);
    auto go = [&](auto kernel, auto params) { hipLaunchKernelGGL(kernel, grid, block, 0, s, params); };
    switch (plan.shape) {
        case gvr_fp8::kAnyShape: go(matmul_kernel<E>, t.p); break;
        case gvr_fp8::kRows: plan.threads == 512 ? go(rows_kernel<E, BYROW, 1, 1, 4, 8>, t.p) : go(rows_kernel<E, BYROW, 1, 1, 4, 16>, t.p); break;
        case gvr_fp8::kRowPairs: go(rows_kernel<E, BYROW, 1, 2, 4, 8>, t.p); break;
        case gvr_fp8::kRows32: go(rows_kernel<E, BYROW, 2, 1, 4, 8>, t.p); break;
        case gvr_fp8::kLow: go(tile_kernel<E, BYROW, 64, 128, 64, 32, 3>, t); break;
        case gvr_fp8::kNarrow: go(tile_kernel<E, BYROW, 128, 64, 64, 32, 3>, t); break;
        case gvr_fp8::kSquare: go(tile_kernel<E, BYROW, 128, 128, 64, 64, 2>, t); break;
        case gvr_fp8::kLarge:
            if constexpr (sizeof(E) == 2) go(tile_kernel<E, BYROW, 256, 256, 128, 64, 2>, t);
            break;
    }
}

template <class E>
gvr_status launch(const TileParams& t, const gvr_fp8::MatmulPlan& plan, void* stream) {
    const hipStream_t s = (hipStream_t)stream;
    t.p.b.rows_per_scale == 1 ? launch_shape<E, true>(t, plan, s) : launch_shape<E, false>(t, plan, s);
    if (t.parts)
        hipLaunchKernelGGL(join_kernel<E>, dim3((unsigned)(t.p.M * t.join_cols)), dim3(gvr_fp8::kThreads), 0, s, t);
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
    for (const bool wide : {false, true}) {   // (float32 results have no 256 x 256 tiles, and may be split otherwise)
        gvr_fp8::Product product;
        const gvr_status fits = gvr_fp8::plan_product(*a, *b, M, N, K, wide, (size_t)-1, &product);
        if (fits != GVR_OK) return fits;
        if (product.workspace > *bytes) *bytes = product.workspace;
    }
    return GVR_OK;
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
    gvr_fp8::Product product;
    const gvr_status fits = gvr_fp8::plan_product(*a, *b, M, N, K, size == 4, ws_bytes, &product);
    if (fits != GVR_OK) return fits;
    const gvr_fp8::MatmulPlan& plan = product.plan;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    TileParams t;
    t.p.a = *a, t.p.b = *b, t.p.out = out;
    if (M == 1) t.p.a.row_stride = 0;   // (as planned)
    if (N == 1) t.p.b.row_stride = 0;
    if (product.copied[0] || product.copied[1]) {
        CopyParams c;
        c.to_stride = product.row_stride, c.K = K, c.chunks = (uint32_t)(product.row_stride / 16);
        const gvr_fp8_matrix* const from[2] = {a, b};
        gvr_fp8_matrix* const to[2] = {&t.p.a, &t.p.b};
        const int64_t rows[2] = {M, N};
        for (int i = 0; i < 2; ++i) {
            c.from[i] = from[i]->codes, c.stride[i] = from[i]->row_stride, c.to[i] = ws + product.at[i];
            c.items[i] = product.copied[i] ? (uint32_t)rows[i] * c.chunks : 0;
            if (product.copied[i]) to[i]->codes = c.to[i], to[i]->row_stride = c.to_stride;
        }
        const uint32_t blocks = (c.items[0] + c.items[1] + gvr_fp8::kThreads - 1) / gvr_fp8::kThreads;
        hipLaunchKernelGGL(copy_kernel, dim3(blocks), dim3(gvr_fp8::kThreads), 0, (hipStream_t)stream, c);
    }
    t.p.M = M, t.p.N = N, t.p.K = K, t.p.out_stride = out_stride;
    t.p.tiles_n = (uint32_t)plan.tiles_n;
    t.parts = plan.splits > 1 ? reinterpret_cast<float*>(ws + product.parts) : nullptr;
    t.tiles_m = (uint32_t)plan.tiles_m;
    t.splits = (uint32_t)plan.splits;
    t.steps = (uint32_t)gvr_fp8::groups_of(K);
    t.join_cols = (uint32_t)((N + 4 * gvr_fp8::kThreads - 1) / (4 * gvr_fp8::kThreads));
    t.steps_each = (uint32_t)plan.steps_each;
    t.band = (uint32_t)plan.band;
    t.quads = gvr_fp8::scale_quads(t.p.a, K, plan.steps_each) && gvr_fp8::scale_quads(t.p.b, K, plan.steps_each);
    return dtype == GVR_BF16 ? launch<__bf16>(t, plan, stream)
           : dtype == GVR_F16 ? launch<_Float16>(t, plan, stream) : launch<float>(t, plan, stream);
}

}  // extern "C"
