// project.cu -- ecasq_project and ecasq_gated: the entry points, and the kernel for few rows of x.
#include <algorithm>

#include "project.cuh"

namespace ecasq {

constexpr int64_t kFewRows = 8;

// A block takes a tile of 32 outputs of 32 rows of x; 128 columns of both at a time lie in shared memory as fp32.
template <typename T, typename S, bool GATED>
__global__ void __launch_bounds__(256) k_project(const __grid_constant__ ProjectArgs a) {
    constexpr int kTile = 32, kCols = 32, kMats = GATED ? 2 : 1;
    __shared__ float xs[kTile][kCols + 1], ws[kMats][kTile][kCols + 1], book[16];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int64_t r0 = (int64_t)blockIdx.x * kTile, i0 = (int64_t)blockIdx.y * kTile;
    if (tid < 16) book[tid] = tid < a.m ? to_f32(static_cast<const T *>(a.levels)[tid]) : 0.f;
    float acc[kMats][2][2] = {};
    for (int64_t k0 = 0; k0 < a.k; k0 += kCols) {
        __syncthreads();
        for (int e = tid; e < kTile * kCols; e += 256) {
            const int i = e / kCols, c = e % kCols;
            const int64_t col = k0 + c;
            xs[i][c] = i0 + i < a.b && col < a.k ? to_f32(static_cast<const T *>(a.x)[(i0 + i) * a.x_row + col]) : 0.f;
            const int w = (int)(col % 128) / 8, at = 16 * (w & 3) + 4 * (w >> 2) + (int)(col % 8) / 2;
            for (int g = 0; g < kMats; g++) {
                float v = 0.f;
                if (r0 + i < a.n && col < a.k) {
                    const int64_t row = r0 + i + g * a.n;
                    const int code = a.codes[row * a.code_row + col / 128 * 64 + at] >> 4 * (col & 1) & 15;
                    v = book[code] * to_f32(static_cast<const S *>(a.scales)[row * a.scale_row + col / a.group]);
                }
                ws[g][i][c] = v;
            }
        }
        __syncthreads();
        for (int c = 0; c < kCols; c++)
            for (int g = 0; g < kMats; g++)
                for (int i = 0; i < 2; i++)
                    for (int j = 0; j < 2; j++) acc[g][i][j] = fmaf(xs[ty + 16 * i][c], ws[g][tx + 16 * j][c], acc[g][i][j]);
    }
    for (int i = 0; i < 2; i++)
        for (int j = 0; j < 2; j++) {
            const int64_t row = r0 + tx + 16 * j, col = i0 + ty + 16 * i;
            if (row >= a.n || col >= a.b) continue;
            float v = acc[0][i][j];
            if (GATED) {
                v = activate(v, a.epi.act) * acc[kMats - 1][i][j];
            } else {
                if (a.epi.bias) v += to_f32(static_cast<const T *>(a.epi.bias)[row]);
                v = activate(v, a.epi.act);
                if (a.epi.residual) v += to_f32(static_cast<const T *>(a.epi.residual)[col * a.epi.residual_row + row]);
            }
            static_cast<T *>(a.y)[col * a.y_row + row] = from_f32<T>(v);
        }
}

template <typename T, typename S> static int launch_project(const ProjectArgs &a, cudaStream_t st) {
    const dim3 grid((unsigned)cdiv(a.n, 32), (unsigned)cdiv(a.b, 32));
    note_launch();
    if (a.gated) k_project<T, S, true><<<grid, 256, 0, st>>>(a);
    else k_project<T, S, false><<<grid, 256, 0, st>>>(a);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

// Both calls: n outputs a row of x, of a matrix with n rows or, gated, 2n.
static int project(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels, int32_t m,
                   const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group, const Epilogue &epi, void *y,
                   int64_t y_row, void *ws, size_t ws_bytes, int32_t *status, bool gated, cudaStream_t st) {
    const bool lost_wait = (type & ECASQ_TEST_LOST_WAIT) != 0;
    type &= ~ECASQ_TEST_LOST_WAIT;
    if (n < 1 || k < 1 || b < 0 || n >= (int64_t)1 << (gated ? 30 : 31) || k >= (int64_t)1 << 31 || b > 8 * 65535 || m < 1 || m > 16 || !type_ok(type) ||
        (scale_type != type && scale_type != ECASQ_F32) || group < 32 || group % 32 || epi.act < ECASQ_ACT_NONE || epi.act > ECASQ_ACT_GELU_TANH)
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!x || !codes || !levels || !scales || !y || !aligned16(codes) || code_row % 16 || code_row < 64 * cdiv(k, 128) || scale_row < cdiv(k, group) ||
        (b > 1 && (x_row < k || y_row < n || (epi.residual && epi.residual_row < n))))
        return ECASQ_EINVAL;
    const ProjectArgs a{x, levels, scales, codes, y, status, x_row, code_row, scale_row, y_row, n, k, b, m, group, type, scale_type, gated, lost_wait, epi};
    if (b > kFewRows) return launch_project_tc(a, ws, ws_bytes, st);
    const bool scales32 = scale_type == ECASQ_F32;
    if (type == ECASQ_F32) return launch_project<float, float>(a, st);
    if (type == ECASQ_F16) return scales32 ? launch_project<__half, float>(a, st) : launch_project<__half, __half>(a, st);
    return scales32 ? launch_project<__nv_bfloat16, float>(a, st) : launch_project<__nv_bfloat16, __nv_bfloat16>(a, st);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

size_t ecasq_workspace_size_project(int64_t b, int64_t n, int64_t k, int32_t type) {
    if (b <= kFewRows || b > 8 * 65535 || n < 1 || k < 1 || k >= (int64_t)1 << 31 || !type_ok(type)) return 0;
    return project_tc_room(b, k, type);
}

int ecasq_project(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels,
                  int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group,
                  const void *bias, int32_t activation, const void *residual, int64_t residual_row, void *y, int64_t y_row, void *ws,
                  size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    return project(x, x_row, type, b, codes, code_row, levels, m, scales, scale_row, scale_type, n, k, group, Epilogue{bias, residual, residual_row, activation}, y,
                   y_row, ws, ws_bytes, status, false, reinterpret_cast<cudaStream_t>(stream));
}

int ecasq_gated(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row, const void *levels,
                int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n, int64_t k, int32_t group,
                int32_t activation, void *y, int64_t y_row, void *ws, size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    return project(x, x_row, type, b, codes, code_row, levels, m, scales, scale_row, scale_type, n, k, group, Epilogue{nullptr, nullptr, 0, activation}, y, y_row, ws,
                   ws_bytes, status, true, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
