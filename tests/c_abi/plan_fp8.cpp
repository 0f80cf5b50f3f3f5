// Prints the plan of each product whose sizes are on standard input ("M N K wide" a
// line), and with an argument, of so many random sizes, the sizes too.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "fp8_plan.h"

using namespace gvr_fp8;

static void print(int64_t M, int64_t N, int64_t K, int wide) {
    const gvr_fp8_matrix m = {nullptr, (K + 15) / 16 * 16, nullptr, groups_of(K), 1, 1, 0};
    MatmulPlan p;
    if (plan_matmul(m, m, M, N, K, wide, (size_t)-1, &p) != GVR_OK) std::exit(1);
    static const char* const names[] = {"any", "rows", "row pairs", "rows32", "low", "narrow", "square", "large"};
    std::printf("%lld %lld %lld %s,%d,%d,%d\n", (long long)M, (long long)N, (long long)K, names[p.shape], p.threads, p.splits > 1, wide);
}

int main(int argc, char** argv) {
    long long M, N, K;
    int wide;
    while (std::scanf("%lld %lld %lld %d", &M, &N, &K, &wide) == 4) print(M, N, K, wide);
    std::mt19937_64 rng(9);
    auto spread = [&](double most) { return (int64_t)std::exp(std::log(most) * (double)(rng() >> 11) * 0x1p-53); };
    for (int i = argc > 1 ? std::atoi(argv[1]) : 0; i > 0; --i) {
        const int64_t m = spread(20000), n = spread(20000), k = spread(20000);
        print(m, n, rng() % 3 ? k : (k + 511) / 512 * 512, (int)(rng() & 1));
    }
}
