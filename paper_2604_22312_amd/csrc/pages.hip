// pages.hip -- block tables, slots and positions from request lengths, behind
// include/gvr_pages.h.
//
// One workgroup adds up the requests, 1024 at a time: the starts of their rows,
// the pages that they need, and, once it is known who is served, the pages given
// back (three scans, each over what the one before decided). Then every place of
// the stack between its old and its new top is one item, and it reads the page
// that is popped there before it writes the one that is pushed there, so pages
// move without an order between items; a request either gets pages or gives some
// back, so tables meet neither. Then every row looks its request up by bisection.
//
// Bound by latency: a step moves a few kilobytes, through lengths, scans, pages and
// table entries one after the other. Small steps run all parts in one workgroup, with
// what the parts hand over in LDS (64 requests of two tokens: 5.0 us, the launch
// included); larger ones add up in one workgroup (300 requests: 5.6 us) and move pages
// (7500: 5) and fill rows (131072: 4.0) in two more kernels. A small step that gives
// 7500 pages back does it in its one workgroup: 14.7.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "gvr_pages.h"
#include "pages_plan.h"
#include "wave_ops.h"

#ifndef DEV
#define DEV __device__ __forceinline__
#endif

namespace {

using gvr_pages::kThreads;
using gvr_pages::kTokenThreads;

struct StepParams {
    gvr_page_pool pool;
    gvr_page_step_args a;
    int32_t* ws;
    int32_t lg_page;
};

// What the parts of a step hand over, of request r: row start (start[R]: the sum
// of all), pages before, tokens after, tokens kept (-1: not served), and the pages
// taken and given back by requests 0 .. r.
struct Hand {
    int32_t *start, *held, *after, *base, *takes, *gives;
    int64_t* total;   // pages taken, pages given back, pages on the stack before
};
DEV Hand hand_over(int32_t* at, int R) {
    const int n = (R + 1 + 3) & ~3;
    Hand h;
    h.total = reinterpret_cast<int64_t*>(at);
    at += 2 * gvr_pages::kHeader;
    h.start = at, h.held = at + n, h.after = at + 2 * n, h.base = at + 3 * n, h.takes = at + 4 * n, h.gives = at + 5 * n;
    return h;
}

// Sum of v over the lanes up to this one, by lane moves.
template <int CTRL, int ROWS>
DEV int64_t moved(int64_t v) {
    const uint32_t lo = (uint32_t)gvr_dev::dpp_i<CTRL, ROWS>(0, (int)(uint32_t)v);
    return (int64_t)((uint64_t)(uint32_t)gvr_dev::dpp_i<CTRL, ROWS>(0, (int)(v >> 32)) << 32 | lo);
}
DEV int64_t wave_scan(int64_t v) {
    v += moved<gvr_dev::kRowShr1, 0xF>(v);
    v += moved<gvr_dev::kRowShr1 + 1, 0xF>(v);
    v += moved<gvr_dev::kRowShr1 + 3, 0xF>(v);
    v += moved<gvr_dev::kRowShr1 + 7, 0xF>(v);
    v += moved<gvr_dev::kRowBcast15, 0xA>(v);
    return v + moved<gvr_dev::kRowBcast31, 0xC>(v);
}

// Sum of v over the threads up to this one; *all: over all of them. Every thread calls it.
DEV int64_t block_scan(int64_t v, int64_t* lds, int64_t* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    v = wave_scan(v);
    __syncthreads();   // (the last scan's numbers are read)
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    int64_t before = 0, sum = 0;
    for (int w = 0; w < waves; ++w) {
        const int64_t u = lds[w];
        before += w < wave ? u : 0;
        sum += u;
    }
    *all = sum;
    return before + v;
}

DEV int32_t pages_of(const StepParams& p, int64_t tokens) {
    return (int32_t)((tokens + p.pool.page_size - 1) >> p.lg_page);
}

DEV void add_up(const StepParams& p, const Hand& h, int64_t* lds) {
    const int R = p.pool.requests;
    const int64_t most = p.pool.width << p.lg_page;
    const int64_t count = R ? min(max((int64_t)p.pool.free_count[0], (int64_t)0), p.pool.pages) : 0;
    int64_t rows = 0, wanted = 0, taken = 0, given = 0;
    for (int r0 = 0; r0 < R; r0 += blockDim.x) {
        const int r = r0 + threadIdx.x;
        const bool live = r < R;
        int64_t ctx = 0, keep = 0, n = 0, all;
        if (live) {
            ctx = min(max((int64_t)p.pool.ctx_len[r], (int64_t)0), most);
            keep = p.a.keep ? min(max((int64_t)p.a.keep[r], (int64_t)0), ctx) : ctx;
            n = max((int64_t)p.a.new_len[r], (int64_t)0);
        }
        const int64_t end = rows + block_scan(n, lds, &all);
        rows += all;
        const int64_t start = end - n, held = pages_of(p, ctx);
        const bool fits = live && end <= p.a.T && keep + n <= most;
        const int64_t more = fits ? max((int64_t)pages_of(p, keep + n) - held, (int64_t)0) : 0;
        const int64_t need = wanted + block_scan(more, lds, &all);
        wanted += all;
        const bool served = fits && (more == 0 || need <= count);
        const int64_t after = served ? keep + n : keep;
        const int64_t takes = taken + block_scan(served ? more : 0, lds, &all);
        taken += all;
        const int64_t gives = given + block_scan(max(held - pages_of(p, after), (int64_t)0), lds, &all);
        given += all;
        if (live) {
            const int32_t first = (int32_t)min(start, p.a.T);
            h.start[r] = first;
            h.held[r] = (int32_t)held;
            h.after[r] = (int32_t)after;
            h.base[r] = served ? (int32_t)keep : -1;
            h.takes[r] = (int32_t)takes;
            h.gives[r] = (int32_t)min(gives, (int64_t)INT32_MAX);   // (more than the stack holds are dropped)
            p.pool.ctx_len[r] = (int32_t)after;
            if (p.a.q_start) p.a.q_start[r] = first;
            if (p.a.taken) p.a.taken[r] = served ? (int32_t)n : 0;
        }
    }
    if (threadIdx.x == 0) {
        h.start[R] = (int32_t)min(rows, p.a.T);
        h.total[0] = taken, h.total[1] = given, h.total[2] = count;
        if (p.a.q_start) p.a.q_start[R] = h.start[R];
        if (R) p.pool.free_count[0] = (int32_t)min(count - taken + given, p.pool.pages);
    }
}

// First r of [0, n) with v[r] > x (n if none), v ascending.
DEV int first_above(const int32_t* v, int n, int32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Places `first`, `first` + step, ... of the stack from its new end up to its old one or its next one, four at a time: all
// loads of the four before their stores (no two places share a number that they read and write).
DEV void move_pages(const StepParams& p, const Hand& h, int64_t first, int64_t step) {
    const int R = p.pool.requests;
    const int64_t taken = h.total[0], given = h.total[1], base = h.total[2] - taken, places = max(taken, given);
    for (int64_t q0 = first; q0 < places; q0 += 4 * step) {
        int32_t got[4], back[4];
        int32_t *to[4], *from[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t q = q0 + u * step, at = base + q;   // of the stack
            to[u] = from[u] = nullptr;
            if (q < taken) {
                const int32_t i = (int32_t)(taken - 1 - q);
                const int r = first_above(h.takes, R, i);
                to[u] = p.pool.block_table + r * p.pool.width + h.held[r] + (i - (r ? h.takes[r - 1] : 0));
                got[u] = p.pool.free_pages[at];
            }
            const int64_t k = given - 1 - q;
            if (q < given && at < p.pool.pages && k < INT32_MAX) {
                const int r = first_above(h.gives, R, (int32_t)k);
                from[u] = p.pool.block_table + r * p.pool.width + pages_of(p, h.after[r]) + ((int32_t)k - (r ? h.gives[r - 1] : 0));
                back[u] = *from[u];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (to[u]) *to[u] = got[u];
            if (from[u]) {
                p.pool.free_pages[base + q0 + u * step] = back[u];
                *from[u] = -1;
            }
        }
    }
}

// starts: h.start + 1, or a copy of it.
DEV void fill_row(const StepParams& p, const Hand& h, const int32_t* starts, int64_t t) {
    const int R = p.pool.requests;
    int32_t pos = 0, see = 0;
    int64_t slot = -1, dense = -1;
    const int r = first_above(starts, R, (int32_t)t);
    const int32_t keep = r < R ? h.base[r] : -1;
    if (keep >= 0) {
        pos = keep + (int32_t)(t - h.start[r]);
        see = pos + 1;
        dense = pos < p.a.ld ? r * p.a.ld + pos : -1;   // (behind them the next request's rows begin)
        if (p.a.slots) {
            const int64_t page = p.pool.block_table[r * p.pool.width + (pos >> p.lg_page)];
            if (page >= 0 && page < (int64_t)1 << (31 - p.lg_page))
                slot = (page << p.lg_page) + (pos & (p.pool.page_size - 1));
        }
    }
    if (p.a.positions) p.a.positions[t] = pos;
    if (p.a.slots) p.a.slots[t] = slot;
    if (p.a.dense) p.a.dense[t] = dense;
    if (p.a.row_len) p.a.row_len[t] = see;
}

__global__ __launch_bounds__(kThreads) void small_step_kernel(StepParams p) {
    __shared__ int64_t sums[kThreads / 64];
    __shared__ __attribute__((aligned(16))) int32_t lds[2 * gvr_pages::kHeader + gvr_pages::kArrays * (gvr_pages::kSmallRequests + 4)];
    const Hand h = hand_over(lds, p.pool.requests);
    add_up(p, h, sums);
    __syncthreads();
    move_pages(p, h, threadIdx.x, blockDim.x);
    __syncthreads();
    for (int64_t t = threadIdx.x; t < p.a.T; t += blockDim.x) fill_row(p, h, h.start + 1, t);
}

__global__ __launch_bounds__(kThreads) void add_up_kernel(StepParams p) {
    __shared__ int64_t sums[kThreads / 64];
    add_up(p, hand_over(p.ws, p.pool.requests), sums);
}

__global__ __launch_bounds__(kTokenThreads) void move_pages_kernel(StepParams p) {
    move_pages(p, hand_over(p.ws, p.pool.requests), (int64_t)blockIdx.x * kTokenThreads + threadIdx.x,
               (int64_t)gridDim.x * kTokenThreads);
}

// The row starts are searched in LDS where they fit: nine loads one after the other from L2 cost 2 us.
__global__ __launch_bounds__(kTokenThreads) void fill_rows_kernel(StepParams p) {
    constexpr int kMost = 2048;
    __shared__ int32_t starts[kMost];
    const int R = p.pool.requests;
    const Hand h = hand_over(p.ws, R);
    const int64_t t = (int64_t)blockIdx.x * kTokenThreads + threadIdx.x;
    const bool here = R <= kMost;
    if (here) {
        for (int r = threadIdx.x; r < R; r += kTokenThreads) starts[r] = h.start[1 + r];
        __syncthreads();
    }
    if (t < p.a.T) fill_row(p, h, here ? starts : h.start + 1, t);
}

}  // namespace

extern "C" {

int64_t gvr_page_step_workspace(int32_t requests) { return gvr_pages::workspace_bytes(requests); }

gvr_status gvr_page_step(const gvr_page_pool* pool, const gvr_page_step_args* args, void* workspace, size_t ws_bytes,
                         void* stream) {
    const gvr_status st = gvr_pages::check(pool, args, workspace, ws_bytes);
    if (st != GVR_OK) return st;
    StepParams p;
    p.pool = *pool;
    p.a = *args;
    p.ws = static_cast<int32_t*>(workspace);
    p.lg_page = 0;
    while ((1 << p.lg_page) < pool->page_size) ++p.lg_page;
    const hipStream_t s = (hipStream_t)stream;
    if (gvr_pages::small_step(pool->requests, args->T)) {
        const int threads = pool->requests <= 256 && args->T <= 256 ? 256 : kThreads;
        hipLaunchKernelGGL(small_step_kernel, dim3(1), dim3(threads), 0, s, p);
    } else {
        hipLaunchKernelGGL(add_up_kernel, dim3(1), dim3(kThreads), 0, s, p);
        const int64_t items = args->T / pool->page_size + pool->requests;   // (pages taken at most; those given back loop)
        const unsigned blocks = (unsigned)(items / (2 * kTokenThreads) + 1 > 512 ? 512 : items / (2 * kTokenThreads) + 1);
        if (pool->requests) hipLaunchKernelGGL(move_pages_kernel, dim3(blocks), dim3(kTokenThreads), 0, s, p);
        if (args->T)
            hipLaunchKernelGGL(fill_rows_kernel, dim3((unsigned)((args->T + kTokenThreads - 1) / kTokenThreads)),
                               dim3(kTokenThreads), 0, s, p);
    }
    return hipGetLastError() == hipSuccess ? GVR_OK : GVR_ERR_HIP;
}

}  // extern "C"
