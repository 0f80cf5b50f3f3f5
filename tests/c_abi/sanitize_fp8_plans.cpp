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

int main() {
    forced_shapes();
    std::printf("ok\n");
}
