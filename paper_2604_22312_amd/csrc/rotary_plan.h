// rotary_plan.h -- argument checks and launch shapes of the rotary and the
// 4-bit cache's token kernels. Plain C++ with no HIP dependency, so the
// library and a sanitizer build on the CPU compile the same code.
#ifndef GVR_ROTARY_PLAN_H
#define GVR_ROTARY_PLAN_H

#include <stddef.h>
#include <stdint.h>

#include "gvr_rotary.h"

namespace gvr_rot {

constexpr int64_t kMaxCount = ((int64_t)1 << 31) - 16;
constexpr int kBlock = 256;
constexpr int64_t kMaxRows = 65535;   // of a launch (blockIdx.y)

// Positions of a workgroup (256 threads) that makes the table: 64, or more where
// a launch's threads would not fit 32 bits (2^30 - 64 positions and more).
inline int table_rows(int64_t n) { return n <= (int64_t)1 << 29 ? 64 : 256; }

inline int dtype_size(int dtype) { return dtype == GVR_F32 ? 4 : (dtype == GVR_BF16 || dtype == GVR_F16) ? 2 : 0; }

// Rows that 16-byte accesses at multiples of 8 elements can serve.
inline bool wide_rows(const gvr_heads& h, int size) {
    const int64_t unit = 16 / size;
    return ((uintptr_t)h.data & 15) == 0 && h.token_stride % unit == 0 && h.head_stride % unit == 0;
}

// GVR_OK if cs can serve heads of D elements (`allowed`: its flags).
inline gvr_status check_cs(const gvr_rope_cs& cs, int D, int allowed) {
    if (cs.rot < 2 || cs.rot > 512 || (cs.rot & 1) || cs.rot > D) return GVR_ERR_INVALID_ARG;
    if (cs.positions < 0 || (cs.positions > 0 && !cs.data) || ((uintptr_t)cs.data & 7)) return GVR_ERR_INVALID_ARG;
    if (cs.flags & ~allowed) return GVR_ERR_INVALID_ARG;
    return GVR_OK;
}

// Table rows that start 16-byte aligned.
inline bool wide_cs(const gvr_rope_cs& cs) { return ((uintptr_t)cs.data & 15) == 0 && cs.rot % 4 == 0; }

// Launch over T tokens x heads x `per_head` items: a thread serves `heads_each`
// heads of one token at the same place in the head (and reads that place's
// cosines once); a launch row (blockIdx.y) takes `tokens` tokens, so that its
// items count in 31 bits.
struct Launch {
    int heads_each, head_groups;
    int64_t tokens, blocks, rows;
};
inline Launch plan_items(int64_t T, int heads, int per_head, int most_heads_each) {
    Launch p;
    // Several heads (both callers: two) where that leaves threads enough to fill
    // the device. One, two,
    // four each (us): rotation of 8192 tokens x 32 heads of 128 28.0, 27.9, 29.6,
    // x 64 heads 40.9, 41.6, 43.6; append of 16384 x 8 heads 22.4, 18.7, 17.8, and
    // read back from HBM 44.1, 42.6, 42.9. Small calls need the threads: 128 x 64
    // heads 4.2 with one, 5.2 with four; an append of 64 x 8 heads 4.2 and 5.5.
    const int64_t fill = (int64_t)256 * 2048, items = T * (int64_t)heads;
    p.heads_each = 1;
    while (p.heads_each < most_heads_each && p.heads_each < heads &&
           items * per_head / (2 * p.heads_each) >= fill)
        p.heads_each *= 2;
    p.head_groups = (heads + p.heads_each - 1) / p.heads_each;
    const int64_t per_token = (int64_t)p.head_groups * per_head;
    p.tokens = kMaxCount / per_token;
    if (p.tokens > T) p.tokens = T;
    if (p.tokens < 1) p.tokens = 1;
    p.blocks = (p.tokens * per_token + kBlock - 1) / kBlock;
    p.rows = (T + p.tokens - 1) / p.tokens;
    return p;
}

}  // namespace gvr_rot

#endif  // GVR_ROTARY_PLAN_H
