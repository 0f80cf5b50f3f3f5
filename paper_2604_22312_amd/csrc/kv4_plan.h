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
constexpr int kJoinThreads = 256;  // of the kernel that joins a row's and head's splits (plans that split have
                                   // few workgroups and so few rows: its launch always fits)
constexpr int64_t kMaxThreads = 0xFFFFFFFF;   // of a launch
constexpr int kMaxSplits = 1024;
constexpr int kMaxBalanced = 2048;  // sequences whose lengths a workgroup adds up
// The model of plan_attention, in tiles' times.
constexpr double kPrologue = 3.0;  // of a workgroup: addresses, queries, the first loads
constexpr double kSecond = 3.0;    // the kernel that joins the splits (and kPart parts read in one)
constexpr double kPart = 4000.0;
constexpr double kApart = 0.1;     // share that a tile takes longer for each halving of the heads read together
constexpr int kCus = 256;          // compute units, each with one workgroup at a time (D = 64: two)
// Query rows of a KV head up to which the few-rows kernel serves (32 contexts of
// 8K, 8 heads of 128: few / many rows 139 / 234 us at 64 rows, 256 / 274 at 128,
// 398 / 348 at 192; 16 of 8K, 4 heads: D = 64, 128 rows 58 / 71, D = 256 149 / 171;
// one of 64K: 128 rows 79 / 82, 192 rows 112 / 104).
constexpr int kFewRows = 128;

// Whether units of workgroups that read the same records are dealt to the eight
// XCDs: evenly, or so many that it comes to little (32 contexts of 8K, 64 rows
// in two tiles: 160 us, and 169 where neighbours go to different XCDs).
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
    int threads;      // of one
    int splits;       // of a context or selection
    int chunk;        // tokens of a split
    bool balanced;    // few rows: the kernel sizes the splits by the contexts' lengths, `units` in all
    int units;        // splits of all sequences
    size_t ws_bytes;
};

// Workspace for `units` splits of `sequences` sequences (no more units than
// sequences: none).
inline size_t partial_bytes(const gvr_kv4_attention_args& a, int max_q, int head_dim, int64_t units) {
    return units > a.sequences ? (size_t)units * max_q * a.q_heads * (head_dim + 2) * 4 + (size_t)a.sequences * 8 : 0;
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
    p.threads = p.many ? 2 * rows_wg : kThreads;
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
        while (splits > 1 && partial_bytes(a, p.max_q, c.head_dim, a.sequences * splits) > ws_bytes) --splits;
        int64_t chunk = ((n + splits - 1) / splits + unit - 1) / unit * unit;
        if (chunk < unit) chunk = unit;
        splits = n > 0 ? (n + chunk - 1) / chunk : 1;
        p.chunk = (int)(chunk > kMaxCount ? kMaxCount / unit * unit : chunk);
        p.splits = (int)splits;
        p.jobs = grid_of((int64_t)a.sequences * c.kv_heads * splits, tiles);
        p.balanced = false;
        p.units = (int)(a.sequences * splits);
        p.ws_bytes = partial_bytes(a, p.max_q, c.head_dim, p.units);
        return p;
    }
    // Heads of a workgroup (all that divide evenly, or fewer with more waves to
    // each) and splits, by a model of the time in tiles: a compute unit takes
    // its workgroups in turn, each for its tiles and for about kPrologue tiles
    // more (addresses, queries, the first loads); splits cost a second kernel,
    // and heads apart cost reads of partly used lines (32 x 32K tokens, 8 heads
    // of 128: 242 us all together, 276 in twos; 1 x 16K: 16.0 and 15.8).
    const int all = log2_of(kWaves);
    int most_hw = 0;
    while (most_hw < all && c.kv_heads % (2 << most_hw) == 0) ++most_hw;
    const int64_t resident = kCus * (c.head_dim == 64 && p.row_tiles == 1 && a.dtype == GVR_BF16 ? 2 : 1);
    double best = -1;
    int64_t splits = 1;
    p.hw_shift = most_hw;
    auto cost = [&](int hw, int64_t s) {
        const int64_t wgs = (int64_t)a.sequences * tiles * (c.kv_heads >> hw) * s;
        const int64_t own = (steps + (kWaves >> hw) * s - 1) / ((kWaves >> hw) * s);
        const double rounds = (double)((wgs + resident - 1) / resident);
        const double parts = (double)a.T * a.q_heads * s;
        return rounds * ((double)own * (1.0 + kApart * (most_hw - hw)) + kPrologue) +
               (s > 1 ? kSecond + 0.01 * s + parts / kPart : 0.0);
    };
    // splits that the workspace holds
    const size_t each = (size_t)a.sequences * p.max_q * a.q_heads * (c.head_dim + 2) * 4, table = (size_t)a.sequences * 8;
    const size_t held = ws_bytes > table && each > 0 ? (ws_bytes - table) / each : 0;
    const int64_t room = held > (size_t)kMaxSplits ? kMaxSplits : (int64_t)held;
    for (int hw = most_hw; hw >= 0; --hw) {
        const int64_t wgs = (int64_t)a.sequences * tiles * (c.kv_heads >> hw);
        const int64_t most = (steps + (kWaves >> hw) - 1) / (kWaves >> hw);
        for (int k = 0; k <= 6; ++k) {   // unsplit, and what fills a quarter of the device to four rounds
            int64_t s = k && wgs > 0 ? resident * (1 << k) / (8 * wgs) : 1;
            s = s > most ? most : s;
            s = s > kMaxSplits ? kMaxSplits : s;
            s = s > room ? room : s;
            if (s < 1) s = 1;
            const double t = cost(hw, s);
            if (best < 0 || t < best) best = t, splits = s, p.hw_shift = hw;
        }
    }
    p.tw_shift = all - p.hw_shift;
    const int64_t unit = (int64_t)kStep << p.tw_shift;
    int64_t chunk = (n + splits - 1) / splits;
    chunk = (chunk + unit - 1) / unit * unit;
    if (chunk < unit) chunk = unit;
    splits = n > 0 ? (n + chunk - 1) / chunk : 1;
    p.chunk = (int)(chunk > kMaxCount ? kMaxCount / unit * unit : chunk);
    p.splits = (int)splits;
    // Contexts of several sequences are rarely of one length: the kernel cuts
    // them so that all the units are about as long.
    p.balanced = splits > 1 && a.sequences > 1 && !a.selection && a.sequences <= kMaxBalanced;
    p.units = (int)(a.sequences * splits);
    const int64_t inner = tiles * (c.kv_heads >> p.hw_shift);
    if (p.balanced) {
        // (what a round of workgroups leaves over is units too)
        const int64_t whole = (p.units * inner + resident - 1) / resident * resident / inner;
        if (whole > p.units && partial_bytes(a, p.max_q, c.head_dim, whole) <= ws_bytes) p.units = (int)whole;
    }
    p.jobs = grid_of(p.units, inner);
    p.ws_bytes = partial_bytes(a, p.max_q, c.head_dim, p.units);
    return p;
}

}  // namespace gvr_kv4

#endif  // GVR_KV4_PLAN_H
