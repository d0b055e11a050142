// epilogue.cuh -- what ecasq_project and ecasq_gated do to a product's fp32 sums before they are rounded.
#pragma once

#include "codes.cuh"

namespace ecasq {

struct Epilogue {
    const void *bias, *residual;  // of x's type, or null
    int64_t residual_row;
    int32_t act;  // ECASQ_ACT_*
};

// Activations in fp32.  The exponentials are the hardware's (2^-22 or so); one that overflows gives the limit, 0.
__device__ __forceinline__ float activate(float v, int act) {
    switch (act) {
        case ECASQ_ACT_RELU: return v <= 0.f ? 0.f : v;  // (NaN stays NaN)
        case ECASQ_ACT_SILU: return __fdividef(v, 1.f + __expf(-v));
        case ECASQ_ACT_GELU: return v * normcdff(v);
        case ECASQ_ACT_GELU_TANH:  // (1 + tanh u) / 2 = 1 / (1 + e^-2u), u = sqrt(2 / pi) (v + 0.044715 v^3)
            return __fdividef(v, 1.f + __expf(-1.5957691216057308f * fmaf(0.044715f * v * v, v, v)));
        default: return v;
    }
}

// N values at once, with one choice of the activation for all of them.
template <int N> __device__ __forceinline__ void activate_all(float (&v)[N], int act) {
    switch (act) {
        case ECASQ_ACT_RELU:
#pragma unroll
            for (int j = 0; j < N; j++) v[j] = activate(v[j], ECASQ_ACT_RELU);
            break;
        case ECASQ_ACT_SILU:
#pragma unroll
            for (int j = 0; j < N; j++) v[j] = activate(v[j], ECASQ_ACT_SILU);
            break;
        case ECASQ_ACT_GELU:
#pragma unroll
            for (int j = 0; j < N; j++) v[j] = activate(v[j], ECASQ_ACT_GELU);
            break;
        case ECASQ_ACT_GELU_TANH:
#pragma unroll
            for (int j = 0; j < N; j++) v[j] = activate(v[j], ECASQ_ACT_GELU_TANH);
            break;
        default: break;
    }
}

}  // namespace ecasq
