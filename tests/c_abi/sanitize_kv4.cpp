// The host-side plans of the 4-bit attention and of the token kernels, on the
// CPU under sanitizers: every plan covers its work and fits 31-bit grids, and
// the workspace that a query asks for gives the call the plan of the query.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "kv4_plan.h"
#include "rotary_plan.h"

#define CHECK(c)                                                       \
    do {                                                               \
        if (!(c)) {                                                    \
            std::printf("failed: %s (line %d)\n", #c, __LINE__);       \
            std::exit(1);                                              \
        }                                                              \
    } while (0)

using namespace gvr_kv4;

static void check_plan(const gvr_kv4_cache& c, const gvr_kv4_attention_args& a, size_t ws) {
    const AttnPlan p = plan_attention(c, a, ws);
    const int64_t n = a.selection ? a.K : a.table_width * c.page_size;
    CHECK(p.ws_bytes <= ws);
    CHECK(p.splits >= 1 && p.splits <= kMaxSplits && p.chunk >= kStep && p.chunk % kStep == 0);
    CHECK((int64_t)p.chunk * p.splits >= n);
    CHECK(p.units >= a.sequences * 1LL);
    CHECK(p.balanced || p.units == (int64_t)a.sequences * p.splits);
    CHECK(!p.balanced || (p.units > a.sequences && a.sequences > 1 && !a.selection));
    CHECK(p.jobs >= 0 && p.max_q >= 0 && p.max_q <= a.T);
    const int G = a.q_heads / c.kv_heads;
    if (p.many) {
        const int rows = c.head_dim == 256 ? 128 : 256;
        CHECK((int64_t)p.tiles * rows >= (int64_t)p.max_q * G && !a.selection);
        CHECK(p.jobs >= (int64_t)a.sequences * c.kv_heads * p.splits * p.tiles);
        CHECK(p.chunk % (rows / 2) == 0 || p.splits == 1);
    } else {
        CHECK((1 << (p.hw_shift + p.tw_shift)) == kWaves && c.kv_heads % (1 << p.hw_shift) == 0);
        CHECK(p.row_tiles == 1 || (p.row_tiles == 2 && c.head_dim != 256));
        const int rows = kRows * p.row_tiles;
        if (a.selection)
            CHECK((int64_t)p.tiles == (int64_t)p.max_q * ((G + rows - 1) / rows));
        else
            CHECK((int64_t)p.tiles * rows >= (int64_t)p.max_q * G);
        CHECK(p.jobs >= (int64_t)p.units * p.tiles * (c.kv_heads >> p.hw_shift));
        CHECK(p.chunk % (kStep << p.tw_shift) == 0);
    }
    if (ws == SIZE_MAX) {
        const AttnPlan q = plan_attention(c, a, p.ws_bytes);
        CHECK(q.splits == p.splits && q.chunk == p.chunk && q.jobs == p.jobs && q.units == p.units && q.many == p.many &&
              q.hw_shift == p.hw_shift && q.balanced == p.balanced && q.ws_bytes == p.ws_bytes);
    }
}

int main() {
    std::mt19937 rng(7);
    auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    const int dims[] = {64, 128, 256};
    static int32_t dummy = 0;
    for (int i = 0; i < 200000; ++i) {
        gvr_kv4_cache c = {nullptr, pick(0, 100000), 1 << pick(0, 8), (int32_t)pick(1, 12), dims[pick(0, 2)], 0};
        gvr_kv4_attention_args a = {};
        a.sequences = (int32_t)(pick(0, 3) ? pick(1, 70) : pick(1, 3000));
        const int64_t nq = pick(0, 3) ? pick(1, 4) : pick(1, 700);
        a.T = a.sequences * nq;
        a.q_heads = c.kv_heads * (int32_t)pick(1, 128);
        a.table_width = pick(0, 1 << pick(0, 14));
        a.dtype = (int32_t)pick(0, 1);
        a.causal = 1;
        if (pick(0, 3) == 0) {
            a.K = (int32_t)pick(1, 2048);
            a.selection = &dummy;
        }
        if (pick(0, 2) == 0) {
            a.q_start = &dummy;
            a.max_q = (int32_t)pick(0, 3 * nq);
        }
        CHECK(check_attention(c, a) == GVR_OK || check_attention(c, a) == GVR_ERR_TOO_LONG);
        if (check_attention(c, a) != GVR_OK) continue;
        check_plan(c, a, SIZE_MAX);
        check_plan(c, a, 0);
        check_plan(c, a, (size_t)pick(0, 1 << 24));
    }
    for (int i = 0; i < 200000; ++i) {
        const int64_t T = pick(1, 1 << pick(0, 24));
        const int heads = (int)pick(1, 300), per = (int)pick(1, 600);
        const gvr_rot::Launch l = gvr_rot::plan_items(T, heads, per, 8);
        CHECK(l.heads_each * l.head_groups >= heads && l.heads_each <= 8);
        CHECK(l.tokens * l.rows >= T && l.tokens * (int64_t)l.head_groups * per <= gvr_rot::kMaxCount);
        CHECK(l.blocks * gvr_rot::kBlock >= l.tokens * (int64_t)l.head_groups * per && l.blocks < (1 << 24));
    }
    std::puts("ok");
    return 0;
}
