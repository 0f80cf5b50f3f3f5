// The plans of the 8-bit matrices and of the page step, on the CPU under
// sanitizers: launches fit, splits cover the sum and their workspace, divisions by
// multiplication are exact, and what a page step hands over fits its workspace.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "fp8_plan.h"
#include "pages_plan.h"

#define CHECK(c)                                                       \
    do {                                                               \
        if (!(c)) {                                                    \
            std::printf("failed: %s (line %d)\n", #c, __LINE__);       \
            std::exit(1);                                              \
        }                                                              \
    } while (0)

using namespace gvr_fp8;

int main() {
    std::mt19937_64 rng(5);
    auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    static uint8_t codes;
    static float scale;
    int split = 0, shapes[8] = {};
    for (int i = 0; i < 300000; ++i) {
        const int64_t M = pick(1, (int64_t)1 << pick(0, 30)), N = pick(1, (int64_t)1 << pick(0, 30)), K = pick(0, (int64_t)1 << pick(0, 22));
        const int64_t blocks = groups_of(K);
        gvr_fp8_matrix a = {nullptr, (K + 15) / 16 * 16, nullptr, blocks, 1, 1, 0};
        gvr_fp8_matrix b = {nullptr, (K + 15) / 16 * 16, nullptr, blocks, 1, pick(0, 1) ? 128 : 1, 0};
        if (pick(0, 9) == 0) a.row_stride += pick(1, 15);
        if (pick(0, 9) == 0) b.scale_row_stride = 1, b.scale_block_stride = N;
        CHECK(check_matmul(&a, &b, M, N, K, false) == GVR_OK);
        const size_t most = pick(0, 3) ? (size_t)-1 : (size_t)pick(0, (int64_t)1 << pick(0, 34));
        MatmulPlan p;
        const gvr_status st = plan_matmul(a, b, M, N, K, pick(0, 1), most, &p);
        if (st == GVR_ERR_TOO_LONG) {
            CHECK((double)M * N > 1e9);
            continue;
        }
        CHECK(st == GVR_OK && p.workgroups >= 1 && p.workgroups * p.threads <= 0xFFFFFFFFll);
        CHECK(p.splits * p.steps_each >= blocks && (p.splits == 1 || (p.splits - 1) * p.steps_each < blocks));
        CHECK(p.workspace <= most && (p.splits == 1) == (p.workspace == 0));
        const Tiles t = tiles_of(p.shape);
        CHECK(p.tiles_m * t.m >= M && (p.tiles_m - 1) * t.m < M && p.tiles_n * t.n >= N && (p.tiles_n - 1) * t.n < N);
        if (p.splits > 1) {
            CHECK(p.steps_each % 4 == 0 && p.shape >= kLow && p.workspace == (size_t)p.splits * M * N * 4);
            CHECK(M * ((N + 4 * kThreads - 1) / (4 * kThreads)) * kThreads <= 0xFFFFFFFFll);   // (the kernel that joins)
            ++split;
        }
        if (p.shape == kRows || p.shape == kRowPairs || p.shape == kRows32) CHECK(p.tiles_m == 1 && M <= t.m);
        if (a.row_stride % 16) CHECK(p.shape == kAnyShape);
        ++shapes[p.shape];
    }
    for (int s = kAnyShape; s <= kLarge; ++s) CHECK(shapes[s] > 100);
    CHECK(split > 1000);
    int copied[3] = {};
    for (int i = 0; i < 300000; ++i) {   // products: copies and parts lie in the workspace, one behind the other
        const int64_t M = pick(1, (int64_t)1 << pick(0, 31)), N = pick(1, (int64_t)1 << pick(0, 31)), K = pick(0, (int64_t)1 << pick(0, 31));
        if (M > kMaxCount || N > kMaxCount || K > kMaxCount) continue;
        const int64_t blocks = groups_of(K);
        gvr_fp8_matrix a = {(uint8_t*)(uintptr_t)(pick(0, 1) ? 4096 : 4097), pick(0, 1) ? K : (K + 15) / 16 * 16, nullptr, blocks, 1, 1, 0};
        gvr_fp8_matrix b = {(uint8_t*)(uintptr_t)4096, pick(0, 1) ? -K : (K + 15) / 16 * 16, nullptr, blocks, 1, 128, 0};
        const size_t most = pick(0, 3) ? (size_t)-1 : (size_t)pick(0, (int64_t)1 << pick(0, 34));
        Product p;
        if (plan_product(a, b, M, N, K, pick(0, 1), most, &p) != GVR_OK) continue;
        CHECK(p.workspace <= most && p.workspace == p.parts + p.plan.workspace && p.parts % 256 == 0);
        size_t end = 0, items = 0;
        for (int k = 0; k < 2; ++k)
            if (p.copied[k]) {
                const int64_t rows = k ? N : M;
                CHECK(p.plan.shape != kAnyShape && p.row_stride >= K && p.row_stride % 16 == 0 && p.at[k] == end && K > 0);
                end += ((size_t)rows * p.row_stride + 255) / 256 * 256;
                items += (size_t)rows * (p.row_stride / 16);
            }
        CHECK(end == p.parts && items < ((size_t)1 << 31));
        if (p.plan.shape != kAnyShape) {   // what is read by 16 bytes is aligned
            CHECK(p.copied[0] || ((uintptr_t)a.codes % 16 == 0 && (M == 1 || a.row_stride % 16 == 0)));
            CHECK(p.copied[1] || N == 1 || (b.row_stride % 16 == 0 && b.row_stride >= 0));
        }
        ++copied[p.copied[0] + p.copied[1]];
    }
    CHECK(copied[0] > 1000 && copied[1] > 1000 && copied[2] > 1000);
    for (int i = 0; i < 2000000; ++i) {
        const uint32_t d = (uint32_t)pick(1, (int64_t)1 << pick(0, 30)), n = (uint32_t)pick(0, 0x7FFFFFFF >> pick(0, 30));
        const Divisor v = divisor(d);
        CHECK(quotient(n, v) == n / d && quotient(n / d * d, v) == n / d);
        if (n >= d) CHECK(quotient(n / d * d - 1, v) == n / d - 1);
    }
    for (int i = 0; i < 200000; ++i) {
        gvr_heads x = {&codes, 1, 1};
        gvr_fp8_heads out = {&codes, 1, 1, &scale, 1, 1};
        const int64_t T = pick(1, (int64_t)1 << pick(0, 31));
        const int H = (int)pick(1, (int64_t)1 << pick(0, 20)), D = (int)pick(1, (int64_t)1 << pick(0, 20));
        const gvr_status st = check_heads(&x, GVR_BF16, T, H, D, nullptr, nullptr, &out, nullptr, T, 0);
        if (st != GVR_OK) {
            CHECK(st == GVR_ERR_TOO_LONG || ((uintptr_t)&codes & 1));
            continue;
        }
        for (const int64_t lanes : {(int64_t)8, (int64_t)16}) {
            const int64_t per = (int64_t)H * groups_of(D) * lanes;
            const HeadsPlan l = plan_heads(T, per);
            CHECK(l.rows <= gvr_rot::kMaxRows && l.tokens * l.rows >= T && l.blocks * kBlock >= l.tokens * per);
            CHECK(l.blocks * kBlock <= (int64_t)1 << 31);   // (so a thread's number is below 2^31, as the division asks)
        }
    }
    CHECK(gvr_pages::workspace_bytes(-1) == -1 && gvr_pages::workspace_bytes(gvr_pages::kMaxRequests + 1) == -1);
    for (int R = 0; R <= gvr_pages::kMaxRequests; R += 1 + R / 7) {
        const int64_t n = (R + 1 + 3) & ~3;   // a part's numbers, R + 1 at most
        CHECK(gvr_pages::workspace_bytes(R) == 8 * gvr_pages::kHeader + 4 * gvr_pages::kArrays * n && n >= R + 1);
    }
    std::printf("ok\n");
}
