// epilogue.cuh -- what ecasq_project and ecasq_gated do to a product's fp32 sums before they are rounded.
#pragma once

#include "codes.cuh"

namespace ecasq {

struct Epilogue {
    const void *bias, *residual;  // of x's type, or null
    int64_t residual_row;
    int32_t act;  // ECASQ_ACT_*
};

// The normal distribution's Phi(v), off by 0.8e-7 at most: erfc(x) = (a1 t + ... + a5 t^5) e^(-x^2), t = 1 / (1 + p x), of Abramowitz and Stegun
// 7.1.26 at x = |v| / sqrt(2).  (CUDA's normcdff is exact to its last bits and took 80 us more for a gated block of 2 x 16384 x 4096 by 2048 rows.)
__device__ __forceinline__ float normal_below(float v) {
    const float x = fabsf(v) * 0.70710678f, t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float q = 0.5f * p * __expf(-x * x);
    return v > 0.f ? 1.f - q : q;
}
// Activations in fp32.  The exponentials are the hardware's (2^-22 or so); one that overflows gives the limit, 0.
__device__ __forceinline__ float activate(float v, int act) {
    switch (act) {
        case ECASQ_ACT_RELU: return v <= 0.f ? 0.f : v;  // (NaN stays NaN)
        case ECASQ_ACT_SILU: return __fdividef(v, 1.f + __expf(-v));
        case ECASQ_ACT_GELU: return v * normal_below(v);
        case ECASQ_ACT_GELU_TANH:  // (1 + tanh u) / 2 = 1 / (1 + e^-2u), u = sqrt(2 / pi) (v + 0.044715 v^3)
            return __fdividef(v, 1.f + __expf(-1.5957691216057308f * fmaf(0.044715f * v * v, v, v)));
        default: return v;
    }
}

}  // namespace ecasq
