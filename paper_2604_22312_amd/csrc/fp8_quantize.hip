// fp8_quantize.hip -- E4M3 codes and a scale per 128 elements, of heads and of
// matrices in both directions, behind include/gvr_fp8.h.
//
// Heads: a thread takes eight elements (or sixteen), so the largest magnitude of a
// block of 128 is four (three) lane exchanges.
//
// Matrices: a workgroup takes 128 x 128 elements, a thread eight columns of eight
// rows, held in registers between the search for the largest magnitudes and the
// codes, so x is read once for both directions. A row's largest is four lane
// exchanges, a column's goes through LDS; the transposed codes are turned in LDS
// and leave as 16 bytes of a column.
//
// Bound by HBM where there is much (8192 x 4096 bfloat16 18.7 us, a copy's rate and a
// little more), the other direction beside it by a chain of load, search, exchange and
// store in each workgroup, all of which run at once (4099 x 4096 float32 26 us, 20 at a copy's
// rate; 4096 x 4096 bfloat16 22, 13 at a copy's rate); else by the launch and the loads
// one after the other: slot, position, table row and element (one key of 128 with its
// rotation 2.2 us on the device, 128 x 64 queries 4.1).

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "gvr_fp8.h"
#include "elem_ops.h"
#include "fp8_codes.h"
#pragma clang force_cuda_host_device begin
#include "fp8_plan.h"
#pragma clang force_cuda_host_device end

namespace {

using namespace gvr_elem;
using namespace gvr_fp8c;
using gvr_fp8::kBlock;
using gvr_fp8::kGroup;

struct HeadsParams {
    const void* x;
    const int64_t* slots;
    const int32_t* positions;
    const float* cs;
    uint8_t* codes;
    float* scale;
    int64_t xt, xh, ct, ch, st, sh;   // strides in elements
    int64_t n_pos, T, tokens, rows;
    int32_t D, rot;
    gvr_fp8::Divisor per_token, per_head;   // threads
    bool inter, pow2;
};

enum { kNoTurn, kHalf, kInter, kAny, kNoTurn16 };   // rotations; kAny also serves rows of any alignment and length

// Where HBM is the bound, six waves to a SIMD, not eight, and codes that go past the caches (4096 x 4096 bfloat16 14.3 -> 12.9
// us, 8192 x 4096 23.7 -> 22.1, 16384 x 4096 40.5 -> 39.3).
template <class E, int MODE, int PER>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(PER == 16 ? 6 : 1, PER == 16 ? 6 : 8)))
void heads_kernel(HeadsParams p) {
    constexpr bool WIDE = MODE != kAny;
    constexpr int LANES = kGroup / PER;   // of a block
    const uint32_t idx = blockIdx.x * (uint32_t)kBlock + threadIdx.x;
    const uint32_t tt = gvr_fp8::quotient(idx, p.per_token), r = idx - tt * p.per_token.d;
    const int h = (int)gvr_fp8::quotient(r, p.per_head), e = PER * (int)(r - (uint32_t)h * p.per_head.d);
    const int64_t t = (int64_t)blockIdx.y * p.tokens + tt;
    if ((int64_t)tt >= p.tokens || t >= p.T) return;   // (all lanes of a block)
    int64_t row = t;
    if (p.slots) {
        row = p.slots[t];
        if (row < 0 || row >= p.rows) return;
    }
    const E* x = static_cast<const E*>(p.x) + t * p.xt + h * p.xh;
    const int half = p.rot / 2, left = p.D - e;   // elements of the head from this lane's first on
    const bool turn = MODE != kNoTurn && e < p.rot;
    const float* cs = nullptr;
    if (turn) {
        const int32_t pos = p.positions[t];
        if (pos >= 0 && pos < p.n_pos) cs = p.cs + (int64_t)pos * p.rot;
    }
    f8 v = {0, 0, 0, 0, 0, 0, 0, 0}, w = v;
    if constexpr (WIDE) {
        if (left > 0) v = load8<true>(x + e);
        if (PER == 16 && left > 8) w = load8<true>(x + e + 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) v[i] = (float)x[e + i];
    }
    if (turn) {
        if constexpr (MODE == kHalf) {
            const bool second = e >= half;
            const int other = second ? e - half : e + half;
            float c[8], s[8];
            load_cs<8, true>(cs, second ? other : e, c, s);
            const f8 o = load8<true>(x + other);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = second ? turn_b(o[i], v[i], c[i], s[i]) : turn_a(v[i], o[i], c[i], s[i]);
        } else if constexpr (MODE == kInter) {
            float c[4], s[4];
            load_cs<4, true>(cs, e / 2, c, s);
            const f8 o = v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = turn_a(o[2 * i], o[2 * i + 1], c[i], s[i]);
                v[2 * i + 1] = turn_b(o[2 * i], o[2 * i + 1], c[i], s[i]);
            }
        } else if constexpr (MODE == kAny) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = e + i;
                if (d < p.rot) {
                    const bool b = p.inter ? d & 1 : d >= half;
                    const int pair = p.inter ? d / 2 : (b ? d - half : d);
                    const float o = (float)x[p.inter ? d ^ 1 : (b ? d - half : d + half)];
                    float c[1], s[1];
                    load_cs<1, false>(cs, pair, c, s);
                    v[i] = b ? turn_b(o, v[i], c[0], s[0]) : turn_a(v[i], o, c[0], s[0]);
                }
            }
        }
    }
    const Scale sc = scale_of(row_largest<LANES>(max(largest(v), largest(w))), p.pow2);
    constexpr bool SHORT = sizeof(E) == 2 && MODE == kNoTurn;   // (a rotated element has 32 bits)
    const uint2 codes = codes_of<SHORT>(v, sc);
    uint8_t* const out = p.codes + row * p.ct + h * p.ch + e;
    if constexpr (PER == 16) {
        const uint2 more = codes_of<SHORT>(w, sc);
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        if (left >= 16) __builtin_nontemporal_store(u4{codes.x, codes.y, more.x, more.y}, reinterpret_cast<u4*>(out));
        else if (left > 0) *reinterpret_cast<uint2*>(out) = codes;
    } else if constexpr (WIDE) {
        if (left > 0) *reinterpret_cast<uint2*>(out) = codes;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) out[i] = (uint8_t)((i < 4 ? codes.x : codes.y) >> (8 * (i & 3)));
    }
    if ((threadIdx.x & (LANES - 1)) == 0) p.scale[row * p.st + h * p.sh + e / kGroup] = sc.scale;
}

template <class E>
gvr_status launch_heads(const HeadsParams& p, const gvr_fp8::HeadsPlan& l, int mode, void* stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks, (unsigned)l.rows), dim3(kBlock), 0, (hipStream_t)stream, p);
    };
    mode == kNoTurn16 ? go(heads_kernel<E, kNoTurn, 16>)
    : mode == kNoTurn ? go(heads_kernel<E, kNoTurn, 8>)
    : mode == kHalf ? go(heads_kernel<E, kHalf, 8>)
    : mode == kInter ? go(heads_kernel<E, kInter, 8>) : go(heads_kernel<E, kAny, 8>);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

struct MatrixParams {
    const void* x;
    int64_t stride, R, C;
    gvr_fp8_matrix out, turned;   // codes NULL: not wanted
    uint32_t col_tiles;
    bool pow2, square, wide_out;   // rows of `out` are 16-byte aligned
};

constexpr int kTurnStride = 144;   // bytes of a column's codes in LDS

// Up to n (8 or 16) bytes of codes to a place of any alignment.
template <int N>
DEV void put_bytes(uint8_t* to, const uint32_t (&v)[N / 4], int64_t n) {
    if (n >= N && ((uintptr_t)to & (N - 1)) == 0) {
        if constexpr (N == 8) *reinterpret_cast<uint2*>(to) = uint2{v[0], v[1]};
        else *reinterpret_cast<uint4*>(to) = uint4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) to[i] = (uint8_t)(v[i / 4] >> (8 * (i & 3)));
    }
}

template <class E, bool WIDE>
__global__ __launch_bounds__(kBlock) void matrix_kernel(MatrixParams p) {
    constexpr bool SHORT = sizeof(E) == 2;
    __shared__ uint32_t tops[16][kGroup];
    __shared__ __attribute__((aligned(16))) uint8_t tile[kGroup * kTurnStride];
    const int64_t r0 = (int64_t)(blockIdx.x / p.col_tiles) * kGroup, c0 = (int64_t)(blockIdx.x % p.col_tiles) * kGroup;
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;   // columns c0 + 8 tc + j of rows r0 + 8 tr + i
    const int64_t left = p.C - c0 - 8 * tc;
    const E* x = static_cast<const E*>(p.x) + (r0 + 8 * tr) * p.stride + c0 + 8 * tc;
    f8 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = f8{0, 0, 0, 0, 0, 0, 0, 0};
        if (r0 + 8 * tr + i < p.R) {
            if (WIDE && left >= 8) {
                v[i] = load8<true>(x + i * p.stride);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) v[i][j] = (float)x[i * p.stride + j];
            }
        }
    }
    Scale whole;
    if (p.square) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, largest(v[i]));
        m = gvr_dev::wave_max_u(m);
        if ((threadIdx.x & 63) == 0) tops[0][threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(tops[0][0], tops[0][1]), max(tops[0][2], tops[0][3]));
        __syncthreads();
        whole = scale_of(m, p.pow2);
        if (threadIdx.x == 0) {
            const int64_t br = r0 / kGroup, bc = c0 / kGroup;
            if (p.out.codes) p.out.scale[br * p.out.scale_row_stride + bc * p.out.scale_block_stride] = whole.scale;
            if (p.turned.codes) p.turned.scale[bc * p.turned.scale_row_stride + br * p.turned.scale_block_stride] = whole.scale;
        }
    }
    uint2 straight[8];
    if (p.out.codes || p.square) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = r0 + 8 * tr + i;
            const Scale s = p.square ? whole : scale_of(row_largest<16>(largest(v[i])), p.pow2);
            straight[i] = codes_of<SHORT>(v[i], s);
            if (p.out.codes && r < p.R && tc == 0 && !p.square)
                p.out.scale[r * p.out.scale_row_stride + c0 / kGroup * p.out.scale_block_stride] = s.scale;
        }
    }
    if (p.out.codes) {
        uint8_t* const to = p.out.codes + (r0 + 8 * tr) * p.out.row_stride + c0 + 8 * tc;
        // Sixteen bytes a lane: neighbours exchange halves of two rows (even lanes keep the first).
        if (p.wide_out && c0 + kGroup <= p.C) {
            const bool odd = tc & 1;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint2 mine = odd ? straight[i + 1] : straight[i], give = odd ? straight[i] : straight[i + 1];
                const uint2 got = {(uint32_t)gvr_dev::dpp_i<gvr_dev::kQuadSwap1>(0, (int)give.x),
                                   (uint32_t)gvr_dev::dpp_i<gvr_dev::kQuadSwap1>(0, (int)give.y)};
                if (r0 + 8 * tr + i + odd < p.R)
                    *reinterpret_cast<uint4*>(to + (i + odd) * p.out.row_stride - 8 * odd) =
                        odd ? uint4{got.x, got.y, mine.x, mine.y} : uint4{mine.x, mine.y, got.x, got.y};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w[2] = {straight[i].x, straight[i].y};
                if (r0 + 8 * tr + i < p.R && left > 0) put_bytes<8>(to + i * p.out.row_stride, w, left);
            }
        }
    }
    if (!p.turned.codes) return;
    if (!p.square) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
            tops[tr][8 * tc + j] = m;
        }
        __syncthreads();
        if (threadIdx.x < kGroup) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = max(m, tops[i][threadIdx.x]);
            const int64_t c = c0 + threadIdx.x;
            tops[0][threadIdx.x] = m;   // (this thread alone reads the column before)
            if (c < p.C)
                p.turned.scale[c * p.turned.scale_row_stride + r0 / kGroup * p.turned.scale_block_stride] =
                    scale_of(m, p.pow2).scale;
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint2 c;
        if (p.square) {
            const uint32_t sel = j & 3;
            uint32_t b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = ((j < 4 ? straight[i].x : straight[i].y) >> (8 * sel)) & 0xFFu;
            c.x = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
            c.y = b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24;
        } else {
            f8 y;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i][j];
            c = codes_of<SHORT>(y, scale_of(tops[0][8 * tc + j], p.pow2));
        }
        *reinterpret_cast<uint2*>(tile + (8 * tc + j) * kTurnStride + 8 * tr) = c;
    }
    __syncthreads();
    // 128 columns of 128 bytes, 16 at a time
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int q = threadIdx.x + k * kBlock, c = q >> 3, o = 16 * (q & 7);
        if (c0 + c < p.C && r0 + o < p.R) {
            const uint4 w = *reinterpret_cast<const uint4*>(tile + c * kTurnStride + o);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
            put_bytes<16>(p.turned.codes + (c0 + c) * p.turned.row_stride + r0 + o, u, p.R - r0 - o);
        }
    }
}

template <class E>
gvr_status launch_matrix(const MatrixParams& p, unsigned blocks, bool wide, void* stream) {
    if (wide)
        hipLaunchKernelGGL((matrix_kernel<E, true>), dim3(blocks), dim3(kBlock), 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL((matrix_kernel<E, false>), dim3(blocks), dim3(kBlock), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // namespace

extern "C" {

gvr_status gvr_fp8_quantize(const gvr_heads* x, int32_t dtype, int64_t T, int32_t H, int32_t D, const int32_t* positions,
                            const gvr_rope_cs* cs, const gvr_fp8_heads* out, const int64_t* slots, int64_t rows,
                            int32_t flags, void* stream) {
    const gvr_status st = gvr_fp8::check_heads(x, dtype, T, H, D, positions, cs, out, slots, rows, flags);
    if (st != GVR_OK) return st;
    if (T == 0 || H == 0) return GVR_OK;
    HeadsParams p;
    p.x = x->data, p.slots = slots, p.positions = positions;
    p.codes = out->codes, p.scale = out->scale;
    p.xt = x->token_stride, p.xh = x->head_stride;
    p.ct = out->token_stride, p.ch = out->head_stride;
    p.st = out->scale_token_stride, p.sh = out->scale_head_stride;
    p.T = T, p.rows = rows, p.D = D;
    p.cs = cs ? cs->data : nullptr, p.n_pos = cs ? cs->positions : 0, p.rot = cs ? cs->rot : 0;
    p.inter = cs && (cs->flags & GVR_ROPE_INTERLEAVED);
    p.pow2 = flags & GVR_FP8_POW2;
    const int size = gvr_rot::dtype_size(dtype);
    const bool wide = gvr_rot::wide_rows(*x, size) && D % 8 == 0 && ((uintptr_t)p.codes & 7) == 0 && p.ct % 8 == 0 &&
                      p.ch % 8 == 0;
    int mode = wide ? kNoTurn : kAny;
    if (cs) {
        if (!wide || !gvr_rot::wide_cs(*cs))
            mode = kAny;
        else if (p.inter)
            mode = p.rot % 8 == 0 ? kInter : kAny;
        else
            mode = p.rot % 16 == 0 ? kHalf : kAny;
    }
    const int64_t blocks = (int64_t)H * gvr_fp8::groups_of(D);
    // Sixteen elements a thread where that leaves threads enough to fill the device (8192 x 4096 bfloat16, not in the caches:
    // 20.7 us when eight took 24.2; from 256 to 2048 rows of 4096 the two differ by 0.5 us at most, either way).
    if (mode == kNoTurn && ((uintptr_t)p.codes & 15) == 0 && p.ct % 16 == 0 && p.ch % 16 == 0 &&
        T * blocks >= (int64_t)256 * 2048 / 8)
        mode = kNoTurn16;
    const int64_t lanes = mode == kNoTurn16 ? 8 : 16;   // threads of a block
    const gvr_fp8::HeadsPlan l = gvr_fp8::plan_heads(T, blocks * lanes);
    p.tokens = l.tokens;
    p.per_token = gvr_fp8::divisor((uint32_t)(blocks * lanes));
    p.per_head = gvr_fp8::divisor((uint32_t)(gvr_fp8::groups_of(D) * lanes));
    return dtype == GVR_BF16 ? launch_heads<__bf16>(p, l, mode, stream)
           : dtype == GVR_F16 ? launch_heads<_Float16>(p, l, mode, stream)
                              : launch_heads<float>(p, l, mode, stream);
}

gvr_status gvr_fp8_quantize_matrix(const void* x, int64_t x_stride, int32_t dtype, int64_t R, int64_t C,
                                   const gvr_fp8_matrix* straight, const gvr_fp8_matrix* transposed, int32_t flags,
                                   void* stream) {
    const gvr_status st = gvr_fp8::check_quantize_matrix(x, dtype, R, C, straight, transposed, flags);
    if (st != GVR_OK) return st;
    if (R == 0 || C == 0 || (!straight && !transposed)) return GVR_OK;
    MatrixParams p;
    const gvr_fp8_matrix none = {nullptr, 0, nullptr, 0, 0, 1, 0};
    p.x = x, p.stride = x_stride, p.R = R, p.C = C;
    p.out = straight ? *straight : none;
    p.turned = transposed ? *transposed : none;
    p.col_tiles = (uint32_t)gvr_fp8::groups_of(C);
    p.pow2 = flags & GVR_FP8_POW2, p.square = flags & GVR_FP8_SQUARE;
    p.wide_out = ((uintptr_t)p.out.codes & 15) == 0 && p.out.row_stride % 16 == 0;
    const unsigned blocks = (unsigned)(gvr_fp8::groups_of(R) * gvr_fp8::groups_of(C));
    const int size = gvr_rot::dtype_size(dtype);
    const bool wide = ((uintptr_t)x & 15) == 0 && x_stride % (16 / size) == 0;
    return dtype == GVR_BF16 ? launch_matrix<__bf16>(p, blocks, wide, stream)
           : dtype == GVR_F16 ? launch_matrix<_Float16>(p, blocks, wide, stream)
                              : launch_matrix<float>(p, blocks, wide, stream);
}

}  // extern "C"
