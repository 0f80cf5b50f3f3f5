// The 4-bit attention's plans at their limits, on the CPU under sanitizers: a
// plan that splits is one whose join fits a launch, and a plan that fits a launch
// counts its rows in 31 bits.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "kv4_plan.h"

#define CHECK(c)                                                       \
    do {                                                               \
        if (!(c)) {                                                    \
            std::printf("failed: %s (line %d)\n", #c, __LINE__);       \
            std::exit(1);                                              \
        }                                                              \
    } while (0)

using namespace gvr_kv4;

int main() {
    std::mt19937_64 rng(11);
    auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    const int dims[] = {64, 128, 256};
    static int32_t dummy = 0;
    int split = 0, many = 0, beyond = 0;
    for (int i = 0; i < 300000; ++i) {
        gvr_kv4_cache c = {nullptr, pick(0, 100000), 1 << pick(0, 8), (int32_t)pick(1, 16), dims[pick(0, 2)], 0};
        gvr_kv4_attention_args a = {};
        a.sequences = (int32_t)pick(1, (int64_t)1 << pick(0, 20));
        a.T = pick(1, (int64_t)1 << pick(0, 30));
        a.q_start = &dummy;
        a.max_q = (int32_t)pick(1, 0x7FFFFFFF >> pick(0, 30));
        a.q_heads = c.kv_heads * (int32_t)pick(1, 128);
        a.table_width = pick(0, (int64_t)1 << pick(0, 20));
        a.causal = 1;
        if (pick(0, 2) == 0) {
            a.K = (int32_t)pick(1, 2048);
            a.selection = &dummy;
        }
        if (check_attention(c, a) != GVR_OK) continue;
        for (size_t ws : {(size_t)0, (size_t)pick(0, 1 << 30), SIZE_MAX}) {
            const AttnPlan p = plan_attention(c, a, ws);
            CHECK(p.threads == (p.many && c.head_dim == 256 ? 256 : 512));
            CHECK(p.ws_bytes <= ws && p.jobs >= 0);
            const bool joins = p.splits > 1 || p.balanced;
            const double rows = (double)a.sequences * p.max_q * a.q_heads;
            CHECK(!joins || rows * kJoinThreads <= (double)kMaxThreads);
            split += joins, many += p.many, beyond += p.jobs > kMaxThreads / p.threads;
            if (p.jobs <= kMaxThreads / p.threads)
                CHECK((int64_t)p.tiles * (p.many ? p.threads / 2 : kRows * p.row_tiles) <= (int64_t)1 << 31);
        }
    }
    CHECK(split > 1000 && many > 1000 && beyond > 1000);
    for (int i = 0; i < 100000; ++i) {   // workgroups of 256 threads that make the rotary table
        const int64_t n = i == 0 ? gvr_rot::kMaxCount : pick(1, (int64_t)1 << pick(0, 31));
        if (n > gvr_rot::kMaxCount) continue;
        const int64_t rows = gvr_rot::table_rows(n);
        CHECK((n + rows - 1) / rows * 256 <= kMaxThreads && rows * 256 < (1 << 24));
    }
    // sizes at which the GPU tests count on two heads a thread
    CHECK(gvr_rot::plan_items(8193, 33, 6, 2).heads_each == 2 && gvr_rot::plan_items(701, 33, 64, 2).heads_each == 2);
    CHECK(gvr_rot::plan_items(4097, 33, 8, 2).heads_each == 2 && gvr_rot::plan_items(4097, 33, 6, 2).heads_each == 1);
    std::puts("ok");
    return 0;
}
