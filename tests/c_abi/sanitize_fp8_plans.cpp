// Plans of 8-bit products that the choosing code does not make, on the CPU under
// sanitizers: what a shape cannot do is an error and no launch.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "fp8_plan.h"

#define CHECK(c)                                                       \
    do {                                                               \
        if (!(c)) {                                                    \
            std::printf("failed: %s (line %d)\n", #c, __LINE__);       \
            std::exit(1);                                              \
        }                                                              \
    } while (0)

using namespace gvr_fp8;

static std::mt19937_64 rng(11);
static int64_t pick(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }

// Any shape with any split on any sizes: refused, or every workgroup begins inside both matrices.
static void forced_shapes() {
    int made[8] = {}, refused[8] = {};
    for (int i = 0; i < 400000; ++i) {
        const int64_t M = pick(1, (int64_t)1 << pick(0, 14)), N = pick(1, (int64_t)1 << pick(0, 14)), K = pick(0, (int64_t)1 << pick(0, 14));
        const Shape shape = (Shape)pick(kAnyShape, kLarge);
        const int64_t splits = pick(0, 1) ? 1 : pick(1, 16);
        const bool wide = pick(0, 1);
        MatmulPlan p;
        if (lay_out(shape, splits, M, N, K, wide, &p) != GVR_OK) {
            ++refused[shape];
            continue;
        }
        ++made[shape];
        const Tiles t = tiles_of(shape);
        CHECK(p.shape == shape && !(shape == kLarge && wide));
        CHECK(p.workgroups == p.tiles_m * p.tiles_n * p.splits);
        CHECK((p.tiles_m - 1) * t.m < M && p.tiles_m * t.m >= M && (p.tiles_n - 1) * t.n < N && p.tiles_n * t.n >= N);
        CHECK((p.splits - 1) * p.steps_each < groups_of(K) || p.splits == 1);
        if (shape == kRows || shape == kRowPairs || shape == kRows32) CHECK((p.workgroups - 1) * t.n < N && M <= t.m);
        if (shape < kLow) CHECK(p.splits == 1);
    }
    for (int s = kAnyShape; s <= kLarge; ++s) CHECK(made[s] > 1000 && refused[s] > 1000 - 1001 * (s >= kLow && s < kLarge));
    // 771 x 531 x 1000 with the kernel of up to 32 rows: 850 workgroups of 16 rows of B, which has 531
    MatmulPlan p;
    for (const int64_t splits : {1, 2, 8}) CHECK(lay_out(kRows32, splits, 771, 531, 1000, true, &p) == GVR_ERR_INVALID_ARG);
    CHECK(lay_out(kRows32, 1, 32, 531, 1000, true, &p) == GVR_OK && p.workgroups == 34);
    CHECK(lay_out(kRows32, 2, 32, 531, 1000, true, &p) == GVR_ERR_INVALID_ARG);
}

// A product with as much workspace as was asked for is planned as with any more, and one with less fits it.
static void exact_workspace() {
    int split = 0, uneven = 0, copied = 0;
    for (int i = 0; i < 300000; ++i) {
        const int64_t M = pick(1, (int64_t)1 << pick(0, 14)), N = pick(1, (int64_t)1 << pick(0, 14)), K = pick(1, (int64_t)1 << pick(0, 14));
        const int64_t blocks = groups_of(K);
        const gvr_fp8_matrix a = {(uint8_t*)(uintptr_t)(pick(0, 3) ? 4096 : 4100), (K + 15) / 16 * 16, nullptr, blocks, 1, 1, 0};
        const gvr_fp8_matrix b = {(uint8_t*)(uintptr_t)4096, pick(0, 3) ? (K + 15) / 16 * 16 : K, nullptr, blocks, 1, 128, 0};
        const bool wide = pick(0, 1);
        Product most, exact, less;
        CHECK(plan_product(a, b, M, N, K, wide, (size_t)-1, &most) == GVR_OK);
        CHECK(plan_product(a, b, M, N, K, wide, most.workspace, &exact) == GVR_OK);
        CHECK(exact.workspace == most.workspace && exact.plan.shape == most.plan.shape && exact.plan.splits == most.plan.splits);
        CHECK(exact.plan.steps_each == most.plan.steps_each && exact.copied[0] == most.copied[0] && exact.copied[1] == most.copied[1]);
        // (what is asked for serves every type of the result)
        Product other;
        CHECK(plan_product(a, b, M, N, K, !wide, (size_t)-1, &other) == GVR_OK);
        const size_t asked = most.workspace > other.workspace ? most.workspace : other.workspace;
        CHECK(plan_product(a, b, M, N, K, wide, asked, &exact) == GVR_OK);
        CHECK(exact.plan.shape == most.plan.shape && exact.plan.splits == most.plan.splits);
        if (most.workspace) {
            CHECK(plan_product(a, b, M, N, K, wide, most.workspace - 1, &less) == GVR_OK && less.workspace < most.workspace);
        }
        split += most.plan.splits > 1;
        uneven += most.plan.splits > 1 && blocks % most.plan.steps_each != 0;
        copied += most.copied[0] || most.copied[1];
    }
    CHECK(split > 10000 && uneven > 2000 && copied > 10000);
}

int main() {
    forced_shapes();
    exact_workspace();
    std::printf("ok\n");
}
