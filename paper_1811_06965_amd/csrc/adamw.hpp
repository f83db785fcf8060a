// adamw.hpp -- the AdamW rule of one fp32 parameter with fp32 states, shared by
// the update of a caller's tensors (adamw.hip) and of a partition (misc.hip).
#pragma once

#include <cmath>

#include "common.hpp"

namespace gp {

struct AdamwScalars {
    float lr, b1, c1, b2, c2, eps;  // c = 1 - b
    float ln_b1, ln_b2;             // step_dev: the bias corrections are computed on the device
    float step_size, inv_root;      // else: lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    unsigned key;                   // of the random bits: the seed's part, and with a host step t's
    const long long* step_dev;
    const float* factor;            // multiplied into every gradient; nullptr: 1; NaN: no update
};
constexpr unsigned KEY_SEED = 0x3C6EF372u, KEY_STEP = 0x1E3779B1u;

inline AdamwScalars adamw_scalars(double lr, double beta1, double beta2, double eps, unsigned seed, long long step,
                                  const long long* step_dev, const float* factor) {
    AdamwScalars s{};
    s.lr = (float)lr;
    s.b1 = (float)beta1;
    s.c1 = (float)(1.0 - beta1);
    s.b2 = (float)beta2;
    s.c2 = (float)(1.0 - beta2);
    s.eps = (float)eps;
    s.key = KEY_SEED * seed;
    s.step_dev = step_dev;
    s.factor = factor;
    if (step_dev) {
        s.ln_b1 = (float)std::log(beta1);
        s.ln_b2 = (float)std::log(beta2);
    } else {
        s.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
        s.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
        s.key += KEY_STEP * (unsigned)step;
    }
    return s;
}

struct AdamwStep {
    float factor, step_size, inv_root;
    unsigned key;
};
// What the whole update shares; false: there is none (a NaN factor).
__device__ __forceinline__ bool adamw_begin(const AdamwScalars& s, AdamwStep& st) {
    st = {s.factor ? s.factor[0] : 1.f, s.step_size, s.inv_root, s.key};
    if (st.factor != st.factor) return false;
    if (s.step_dev) {
        const long long t = s.step_dev[0];
        st.step_size = s.lr / -expm1f((float)t * s.ln_b1);
        st.inv_root = 1.f / sqrtf(-expm1f((float)t * s.ln_b2));
        st.key += KEY_STEP * (unsigned)t;
    }
    return true;
}
// The new first moment and second moment from the gradient; every product and sum is rounded by
// itself, in the order of the formulas, so that an update is the same bits wherever
// it is compiled.
__device__ __forceinline__ void adamw_moments(float g, float& m, float& v, const AdamwScalars& s, const AdamwStep& st) {
#pragma clang fp contract(off)
    g = g * st.factor;
    m = m * s.b1 + g * s.c1;
    v = v * s.b2 + g * g * s.c2;
}
// The new parameter; keep = 1 - lr weight_decay.
__device__ __forceinline__ float adamw_param(float p, float m, float v, float keep, const AdamwScalars& s,
                                             const AdamwStep& st) {
#pragma clang fp contract(off)
    return p * keep - st.step_size * m / (sqrtf(v) * st.inv_root + s.eps);
}

// step[0] += 1 on the stream, unless the factor says that there is no update.
gp_status adamw_advance(long long* step, const float* factor, hipStream_t st);

} // namespace gp
