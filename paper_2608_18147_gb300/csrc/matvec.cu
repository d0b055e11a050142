// matvec.cu -- products with a matrix of 4-bit codes (ecasq_pack, ecasq_matvec).
#include <algorithm>

#include "codes.cuh"

namespace ecasq {

// Position of word w of a 128-column block among its sixteen stored words.
__host__ __device__ constexpr int packed_word(int w) { return 4 * (w & 3) + (w >> 2); }

// One thread a word of eight codes.
__global__ void __launch_bounds__(256) k_pack(const uint8_t *__restrict__ idx, int64_t idx_row, int64_t n, int64_t k,
                                              uint8_t *__restrict__ codes, int64_t code_row, int64_t words) {
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n * words; i += stride) {
        const int64_t r = i / words, w = i % words;
        uint32_t v = 0;
        for (int j = 0; j < 8; j++) {
            const int64_t c = 8 * w + j;
            if (c < k) v |= (uint32_t)(idx[r * idx_row + c] & 15) << (4 * j);
        }
        const int64_t at = (w & ~(int64_t)15) + packed_word((int)(w & 15));
        *reinterpret_cast<uint32_t *>(codes + r * code_row + 4 * at) = v;
    }
}

struct MatvecArgs {
    const void *x, *levels, *scales;
    const uint8_t *codes;
    void *y;
    int64_t x_row, code_row, scale_row, y_row, n, k;
    int b, m, group;
};

// One warp a row and eight rows of x, each lane every 32nd column.
template <typename T, typename S>
__global__ void __launch_bounds__(256) k_matvec(MatvecArgs a) {
    const int lane = threadIdx.x & 31, i0 = 8 * blockIdx.y, nb = min(8, a.b - i0);
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (r >= a.n) return;
    const T *x = static_cast<const T *>(a.x) + i0 * a.x_row, *levels = static_cast<const T *>(a.levels);
    const S *scales = static_cast<const S *>(a.scales) + r * a.scale_row;
    const uint32_t *row = reinterpret_cast<const uint32_t *>(a.codes + r * a.code_row);
    float acc[8] = {};
    for (int64_t c = lane; c < a.k; c += 32) {
        const int64_t w = c >> 3;
        const int code = row[(w & ~(int64_t)15) + packed_word((int)(w & 15))] >> (4 * (c & 7)) & 15;
        const float v = code < a.m ? to_f32(levels[code]) * to_f32(scales[c / a.group]) : 0.f;
        for (int i = 0; i < 8; i++)
            if (i < nb) acc[i] = fmaf(v, to_f32(x[i * a.x_row + c]), acc[i]);
    }
    for (int i = 0; i < 8; i++) {
        float s = acc[i];
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0 && i < nb) static_cast<T *>(a.y)[(i0 + i) * a.y_row + r] = from_f32<T>(s);
    }
}

template <typename T>
static void launch_matvec(const MatvecArgs &a, bool scales32, cudaStream_t st) {
    const dim3 grid((unsigned)cdiv(a.n, 8), (unsigned)cdiv(a.b, 8));
    if (scales32) k_matvec<T, float><<<grid, 256, 0, st>>>(a);
    else k_matvec<T, T><<<grid, 256, 0, st>>>(a);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

int ecasq_pack(const uint8_t *idx, int64_t idx_row, int64_t n, int64_t k, uint8_t *codes, int64_t code_row,
               ecasq_stream_t stream) {
    if (!idx || !codes || n < 1 || k < 1 || n >= (int64_t)1 << 31 || k >= (int64_t)1 << 31 || idx_row < k ||
        code_row < 64 * cdiv(k, 128) || code_row % 16 || !aligned16(codes))
        return ECASQ_EINVAL;
    const int64_t words = 16 * cdiv(k, 128);
    note_launch();
    k_pack<<<(unsigned)std::min<int64_t>(cdiv(n * words, 256), 152 * 8), 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(
        idx, idx_row, n, k, codes, code_row, words);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

int ecasq_matvec(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row,
                 const void *levels, int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n,
                 int64_t k, int32_t group, void *y, int64_t y_row, ecasq_stream_t stream) {
    if (n < 1 || k < 1 || b < 0 || n >= (int64_t)1 << 31 || k >= (int64_t)1 << 31 || b > 8 * 65535 || m < 1 || m > 16 ||
        !type_ok(type) || (scale_type != type && scale_type != ECASQ_F32) || group < 32 || group % 32)
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!x || !codes || !levels || !scales || !y || !aligned16(codes) || code_row % 16 || code_row < 64 * cdiv(k, 128) ||
        scale_row < cdiv(k, group) || (b > 1 && (x_row < k || y_row < n)))
        return ECASQ_EINVAL;
    const MatvecArgs a{x, levels, scales, codes, y, x_row, code_row, scale_row, y_row, n, k, (int)b, m, group};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool scales32 = scale_type == ECASQ_F32;
    note_launch();
    if (type == ECASQ_F32) launch_matvec<float>(a, scales32, st);
    else if (type == ECASQ_F16) launch_matvec<__half>(a, scales32, st);
    else launch_matvec<__nv_bfloat16>(a, scales32, st);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

}  // extern "C"
