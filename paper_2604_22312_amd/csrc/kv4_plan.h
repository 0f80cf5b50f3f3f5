// kv4_plan.h -- the 4-bit cache's record layout, argument checks and the
// attention's launch plan. Plain C++ with no HIP dependency, so the library
// and a sanitizer build on the CPU compile the same code.
#ifndef GVR_KV4_PLAN_H
#define GVR_KV4_PLAN_H

#include <stddef.h>
#include <stdint.h>

#include "gvr_kv4.h"
#include "rotary_plan.h"

namespace gvr_kv4 {

using gvr_rot::kMaxCount;

inline int64_t record_bytes(int kv_heads, int head_dim) {
    if (kv_heads < 1 || kv_heads > 1024 || !(head_dim == 64 || head_dim == 128 || head_dim == 256)) return -1;
    return (int64_t)kv_heads * head_dim * 17 / 16;
}

inline int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

// The cache's sizes; its pointer only when slots could be touched.
inline gvr_status check_cache(const gvr_kv4_cache* c, bool need_data) {
    if (!c || record_bytes(c->kv_heads, c->head_dim) < 0 || c->reserved != 0) return GVR_ERR_INVALID_ARG;
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) || c->pages < 0)
        return GVR_ERR_INVALID_ARG;
    if (c->pages > kMaxCount || c->pages * c->page_size > kMaxCount) return GVR_ERR_TOO_LONG;
    if (need_data && c->pages > 0 && !c->data) return GVR_ERR_INVALID_ARG;
    if ((uintptr_t)c->data & 15) return GVR_ERR_INVALID_ARG;
    return GVR_OK;
}

// The attention's sizes (pointers are the caller's part).
inline gvr_status check_attention(const gvr_kv4_cache& c, const gvr_kv4_attention_args& a) {
    if (a.T < 0 || a.sequences < 0 || a.table_width < 0 || a.q_heads < 1 || a.reserved != 0) return GVR_ERR_INVALID_ARG;
    if (a.q_heads % c.kv_heads || a.q_heads / c.kv_heads > 128) return GVR_ERR_INVALID_ARG;
    if (!(a.dtype == GVR_BF16 || a.dtype == GVR_F16) || !(a.causal == 0 || a.causal == 1)) return GVR_ERR_INVALID_ARG;
    if (!(a.scale == a.scale) || a.scale - a.scale != 0.f) return GVR_ERR_INVALID_ARG;   // finite
    if ((a.q_token_stride | a.q_head_stride) & 7) return GVR_ERR_INVALID_ARG;
    if (a.selection && a.K < 1) return GVR_ERR_INVALID_ARG;
    if (a.q_start ? a.max_q < 0 : (a.sequences > 0 && a.T % a.sequences)) return GVR_ERR_INVALID_ARG;
    if (a.T > kMaxCount || a.table_width > kMaxCount || a.table_width * c.page_size > kMaxCount) return GVR_ERR_TOO_LONG;
    return GVR_OK;
}

constexpr int kRows = 16;          // query rows of a wave
constexpr int kStep = 32;          // tokens of a wave's step
constexpr int kWaves = 8;          // of a workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kSlots = 4096;       // tokens whose slots a workgroup holds in LDS
constexpr int kMaxSplits = 1024;
constexpr int kCus = 256;          // compute units, each with one workgroup at a time (D = 64: two)
constexpr int kMinTiles = 4;       // fewest tiles of a workgroup worth another split
constexpr int kFewRows = 64;       // query rows of a KV head up to which the few-rows kernel serves
constexpr int kShort = 64;         // steps of a context that one workgroup takes, so that no second kernel runs

// Whether units of workgroups that read the same records are dealt to the eight
// XCDs: evenly, or so many that it comes to little.
inline bool by_xcd(int64_t units) { return units % 8 == 0 || units >= 64; }
inline int64_t grid_of(int64_t units, int64_t inner) { return (by_xcd(units) ? (units + 7) / 8 * 8 : units) * inner; }

struct AttnPlan {
    int max_q;        // query tokens of a sequence
    bool many;        // the kernel for many query rows
    int row_tiles;    // few rows: tiles of kRows of a wave
    int tiles;        // tiles of rows of a sequence and KV head (a workgroup's)
    int hw_shift;     // log2 of the KV heads of a workgroup
    int tw_shift;     // log2 of the waves that share a head's steps
    int64_t jobs;     // workgroups
    int splits;       // of a context or selection
    int chunk;        // tokens of a split
    size_t ws_bytes;
};

inline size_t partial_bytes(int64_t T, int q_heads, int head_dim, int64_t splits) {
    return splits > 1 ? (size_t)T * q_heads * splits * (head_dim + 2) * 4 : 0;
}

inline AttnPlan plan_attention(const gvr_kv4_cache& c, const gvr_kv4_attention_args& a, size_t ws_bytes) {
    AttnPlan p;
    const int G = a.q_heads / c.kv_heads;
    p.max_q = a.q_start ? a.max_q : (int)(a.T / a.sequences);
    if (p.max_q > a.T) p.max_q = (int)a.T;
    // Many rows of a KV head that see (nearly) the same tokens: V is unpacked
    // once for all of them.
    p.many = !a.selection && (int64_t)p.max_q * G > kFewRows;
    const int rows_wg = c.head_dim == 256 ? 128 : 256;
    // rows that share their tokens; two tiles a wave read K and V once for both
    const int64_t together = a.selection ? G : (int64_t)p.max_q * G;
    p.row_tiles = together > kRows && c.head_dim != 256 ? 2 : 1;
    const int rows = p.many ? rows_wg : p.row_tiles * kRows;
    const int64_t tiles = a.selection ? (int64_t)p.max_q * ((G + rows - 1) / rows) : (together + rows - 1) / rows;
    p.tiles = (int)(tiles > kMaxCount ? kMaxCount : tiles);
    const int64_t n = a.selection ? a.K : a.table_width * c.page_size;
    const int64_t steps = (n + kStep - 1) / kStep;
    const int64_t units = (int64_t)a.sequences * tiles;
    if (p.many) {
        p.hw_shift = p.tw_shift = 0;
        const int64_t unit = rows_wg / 2, wgs = units * c.kv_heads;
        int64_t splits = wgs > 0 && wgs < kCus ? kCus / wgs : 1;
        const int64_t most = (n + 4 * unit - 1) / (4 * unit);   // four tiles at least
        splits = splits > most ? most : splits;
        if (splits < 1) splits = 1;
        while (splits > 1 && partial_bytes(a.T, a.q_heads, c.head_dim, splits) > ws_bytes) --splits;
        int64_t chunk = ((n + splits - 1) / splits + unit - 1) / unit * unit;
        if (chunk < unit) chunk = unit;
        splits = n > 0 ? (n + chunk - 1) / chunk : 1;
        p.chunk = (int)(chunk > kMaxCount ? kMaxCount / unit * unit : chunk);
        p.splits = (int)splits;
        p.jobs = grid_of((int64_t)a.sequences * c.kv_heads * splits, tiles);
        p.ws_bytes = partial_bytes(a.T, a.q_heads, c.head_dim, splits);
        return p;
    }
    // KV heads of a workgroup: all that divide evenly (a record's parts are then
    // read together), fewer, with more waves to each, while that spares splits
    // and the contexts still last for several tiles.
    const int all = log2_of(kWaves);
    p.hw_shift = 0;
    while (p.hw_shift < all && c.kv_heads % (2 << p.hw_shift) == 0) ++p.hw_shift;
    auto jobs = [&](int hw) { return units * (c.kv_heads >> hw); };
    auto tiles_of = [&](int hw) { return (steps + (kWaves >> hw) - 1) / (kWaves >> hw); };
    while (p.hw_shift > 0 && jobs(p.hw_shift) < kCus && tiles_of(p.hw_shift - 1) >= kMinTiles &&
           (jobs(p.hw_shift - 1) >= kCus / 2 || steps <= kShort))
        --p.hw_shift;
    p.tw_shift = all - p.hw_shift;
    const int64_t fill = c.head_dim == 64 ? 2 * kCus : kCus;
    int64_t splits = 1;
    if (jobs(p.hw_shift) < kCus && steps > kShort) {
        splits = jobs(p.hw_shift) > 0 ? (fill + jobs(p.hw_shift) - 1) / jobs(p.hw_shift) : 1;
        const int64_t most = (tiles_of(p.hw_shift) + kMinTiles - 1) / kMinTiles;
        splits = splits > most ? most : splits;
    }
    if (splits > kMaxSplits) splits = kMaxSplits;
    while (splits > 1 && partial_bytes(a.T, a.q_heads, c.head_dim, splits) > ws_bytes) --splits;
    const int64_t unit = (int64_t)kStep << p.tw_shift;
    int64_t chunk = (n + splits - 1) / splits;
    chunk = (chunk + unit - 1) / unit * unit;
    if (chunk < unit) chunk = unit;
    splits = n > 0 ? (n + chunk - 1) / chunk : 1;
    p.chunk = (int)(chunk > kMaxCount ? kMaxCount / unit * unit : chunk);
    p.splits = (int)splits;
    p.jobs = grid_of((int64_t)a.sequences * splits, tiles * (c.kv_heads >> p.hw_shift));
    p.ws_bytes = partial_bytes(a.T, a.q_heads, c.head_dim, splits);
    return p;
}

}  // namespace gvr_kv4

#endif  // GVR_KV4_PLAN_H
