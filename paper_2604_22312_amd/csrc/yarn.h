// yarn.h -- the RoPE / YaRN angles theta'_i shared by the static prior and the
// rotary table, and the check of their parameters.
#ifndef GVR_YARN_H
#define GVR_YARN_H

#include <hip/hip_runtime.h>

#include <math.h>

#include "gvr_rope_prior.h"

#ifndef DEV
#define DEV __device__ __forceinline__
#endif

namespace gvr_yarn {

constexpr int kMaxPairs = 256;               // d <= 512

struct RopeArgs {
    int d;
    int orig_ctx;
    double base, scale, beta_fast, beta_slow;
};

// theta'_i of one rotary pair (YaRN ramp over the pair index).
DEV double yarn_angle(int i, const RopeArgs& a) {
#pragma clang fp contract(off)
    const double two_pi = 6.283185307179586;
    const double ln_base = log(a.base);
    const double x_fast = a.d * log(a.orig_ctx / (two_pi * a.beta_fast)) / (2.0 * ln_base);
    const double x_slow = a.d * log(a.orig_ctx / (two_pi * a.beta_slow)) / (2.0 * ln_base);
    const double lo = fmax(floor(x_fast), 0.0);
    const double hi = fmin(ceil(x_slow), (double)(a.d - 1));
    const double theta = pow(a.base, -2.0 * i / a.d);
    const double gamma = fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
    return theta * (1.0 - gamma) + (theta / a.scale) * gamma;
}

inline bool finite_pos(double v) { return isfinite(v) && v > 0.0; }

inline gvr_status read_params(const gvr_rope_params* p, RopeArgs* a) {
    gvr_rope_params d;
    if (!p) {
        gvr_rope_params_default(&d);
        p = &d;
    }
    if (p->d_rope < 2 || p->d_rope > 2 * kMaxPairs || (p->d_rope & 1)) return GVR_ERR_INVALID_ARG;
    if (p->orig_ctx < 1) return GVR_ERR_INVALID_ARG;
    if (!isfinite(p->base) || p->base <= 1.0) return GVR_ERR_INVALID_ARG;
    if (!finite_pos(p->scale) || !finite_pos(p->beta_fast) || !finite_pos(p->beta_slow)) return GVR_ERR_INVALID_ARG;
    a->d = p->d_rope;
    a->orig_ctx = p->orig_ctx;
    a->base = p->base;
    a->scale = p->scale;
    a->beta_fast = p->beta_fast;
    a->beta_slow = p->beta_slow;
    return GVR_OK;
}

}  // namespace gvr_yarn

#endif  // GVR_YARN_H
