// norm.cu -- root-mean-square norm with the residual's addition, rounded to the input's type or coded to 8 bits (ecasq_norm).
#include <cuda_fp8.h>

#include <algorithm>

#include "codes.cuh"

namespace ecasq {

struct NormArgs {
    const void *x, *residual, *weight;
    void *y, *sum;
    float *scales;
    int64_t x_row, residual_row, y_row, sum_row, scale_row, b, k, group, groups;
    float eps;
};

constexpr int kNormThreads = 256;

// The larger of two values that are not negative; NaN is above all, as its bits are.
__device__ __forceinline__ float above(float v, float w) { return __uint_as_float(max(__float_as_uint(v), __float_as_uint(w))); }

// The sum (MAX: the maximum) over a block, for every thread.
template <bool MAX> __device__ __forceinline__ float over_block(float v) {
    __shared__ float part[kNormThreads / 32];
    for (int o = 16; o; o >>= 1) {
        const float w = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? above(v, w) : v + w;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < kNormThreads / 32; i++) v = MAX ? above(v, part[i]) : v + part[i];
    return v;
}

// A block a row, which it reads once for the mean, and again for what it writes.
template <typename T, typename W> __global__ void __launch_bounds__(kNormThreads) k_norm(const __grid_constant__ NormArgs a) {
    for (int64_t row = blockIdx.x; row < a.b; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_row, *residual = static_cast<const T *>(a.residual) + (a.residual ? row * a.residual_row : 0);
        T *sum = static_cast<T *>(a.sum) + (a.sum ? row * a.sum_row : 0);
        const W *weight = static_cast<const W *>(a.weight);
        auto total = [&](int64_t c) { return a.residual ? from_f32<T>(to_f32(x[c]) + to_f32(residual[c])) : x[c]; };
        float squares = 0.f;
        for (int64_t c = threadIdx.x; c < a.k; c += kNormThreads) {
            const T s = total(c);
            squares = fmaf(to_f32(s), to_f32(s), squares);
            if (a.sum) sum[c] = s;
        }
        const float r = 1.f / sqrtf(over_block<false>(squares) / (float)a.k + a.eps);
        auto normed = [&](int64_t c) { return to_f32(a.sum ? sum[c] : total(c)) * r * to_f32(weight[c]); };  // (its own thread wrote sum[c])
        if (!a.group) {
            T *y = static_cast<T *>(a.y) + row * a.y_row;
            for (int64_t c = threadIdx.x; c < a.k; c += kNormThreads) y[c] = from_f32<T>(normed(c));
            continue;
        }
        uint8_t *y = static_cast<uint8_t *>(a.y) + row * a.y_row;
        for (int64_t g = 0; g < a.groups; g++) {
            const int64_t first = g * a.group + (threadIdx.x - g * a.group % kNormThreads + kNormThreads) % kNormThreads, end = min(a.k, (g + 1) * a.group);
            float most = 0.f;
            for (int64_t c = first; c < end; c += kNormThreads) most = above(most, fabsf(normed(c)));
            most = over_block<true>(most) / 448.f;
            const float scale = most == 0.f ? 1.f : most;
            if (threadIdx.x == 0) a.scales[row * a.scale_row + g] = scale;
            for (int64_t c = first; c < end; c += kNormThreads) y[c] = __nv_cvt_float_to_fp8(normed(c) / scale, __NV_SATFINITE, __NV_E4M3);
        }
    }
}

template <typename T, typename W> static int launch_norm(const NormArgs &a, cudaStream_t st) {
    note_launch();
    k_norm<T, W><<<(unsigned)std::min<int64_t>(a.b, 152 * 16), kNormThreads, 0, st>>>(a);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

}  // namespace ecasq

using namespace ecasq;

extern "C" int ecasq_norm(const void *x, int64_t x_row, int32_t type, int64_t b, int64_t k, const void *residual, int64_t residual_row,
                          const void *weight, int32_t weight_type, float eps, int64_t group, void *y, int64_t y_row, void *sum,
                          int64_t sum_row, float *scales, int64_t scale_row, ecasq_stream_t stream) {
    if (b < 0 || k < 1 || b >= (int64_t)1 << 31 || !type_ok(type) || (weight_type != type && weight_type != ECASQ_F32) || !(eps >= 0.f) || group < 0 ||
        k >= (int64_t)1 << 31 || (group < k && group % 16))
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    const int64_t groups = group ? cdiv(k, group) : 0;
    if (!x || !weight || !y || (sum && !residual) || (group && (!scales || (b > 1 && scale_row < groups))) ||
        (b > 1 && (x_row < k || y_row < k || (residual && residual_row < k) || (sum && sum_row < k))))
        return ECASQ_EINVAL;
    const NormArgs a{x, residual, weight, y, sum, scales, x_row, residual_row, y_row, sum_row, scale_row, b, k, group, groups, eps};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool weight32 = weight_type == ECASQ_F32;
    if (type == ECASQ_F32) return launch_norm<float, float>(a, st);
    if (type == ECASQ_F16) return weight32 ? launch_norm<__half, float>(a, st) : launch_norm<__half, __half>(a, st);
    return weight32 ? launch_norm<__nv_bfloat16, float>(a, st) : launch_norm<__nv_bfloat16, __nv_bfloat16>(a, st);
}
