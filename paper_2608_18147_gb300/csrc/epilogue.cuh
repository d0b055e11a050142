// epilogue.cuh -- what ecasq_project and ecasq_gated do to a product's fp32 sums before they are rounded.
#pragma once

#include "codes.cuh"

namespace ecasq {

struct Epilogue {
    const void *bias, *residual;  // of x's type, or null
    int64_t residual_row;
    int32_t act;  // ECASQ_ACT_*
};

// The normal distribution's Phi(v), off by 2^-23 at most, and for v >= -12 by (2^-21 + v^2 2^-23) of itself at most.  Near zero 1/2 + v P(v^2); elsewhere the tail,
// e^(-v^2 / 2) Q(1 / (1 + 0.32 |v|)).  P and Q are minimax polynomials found by Remez' exchange: P on |v| <= 1.25 (4e-9 of Phi), Q on 1.25 <= |v| <= 14
// (1.4e-7 of the tail).  A gated block of 2 x 16384 x 4096 by 2048 rows takes 470 us with it.  (With Abramowitz and Stegun's 7.1.26, whose error is bounded against 1 alone
// and which was off by 2.4e-7 in fp32 and by 0.4 % of Phi at v = -5, 455 us; with CUDA's normcdff 80 us more than that.)
__device__ __forceinline__ float normal_below(float v) {
    const float x = fabsf(v), y = v * v, t = __fdividef(1.f, fmaf(0.32f, x, 1.f));
    float p = fmaf(y, -6.83135290e-6f, 1.11127045e-4f), q = fmaf(t, -0.0797425291f, 0.173089872f);
    p = fmaf(y, p, -1.18395555e-3f);
    p = fmaf(y, p, 9.97234950e-3f);
    p = fmaf(y, p, -0.0664902212f);
    p = fmaf(y, p, 0.398942277f);
    q = fmaf(t, q, 0.0160783282f);
    q = fmaf(t, q, 0.139521287f);
    q = fmaf(t, q, 0.122674665f);
    q = fmaf(t, q, 0.128200076f);
    q = fmaf(t, q, -2.42528593e-5f) * exp2f(-0.72134752f * y);
    return x < 1.25f ? fmaf(v, p, 0.5f) : v > 0.f ? 1.f - q : q;
}
// Activations in fp32.  The exponentials are the hardware's, off by 2^-21 + |u| 2^-23 of themselves for e^u or so; one that overflows gives the limit, 0.
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
