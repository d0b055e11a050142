// matvec.cu -- products with a matrix of 4-bit codes (ecasq_pack, ecasq_matvec): the packing, the kernel for 16-bit types.
#include <algorithm>

#include "matvec16.cuh"

namespace ecasq {

// Position of word w of a 128-column block among its sixteen stored words.
__host__ __device__ constexpr int packed_word(int w) { return 4 * (w & 3) + (w >> 2); }

// The low four bits of four bytes, side by side.
__device__ __forceinline__ uint32_t four_codes(uint32_t w) {
    w &= 0x0f0f0f0fu;
    w = (w | w >> 4) & 0x00ff00ffu;
    return (w | w >> 8) & 0xffffu;
}

// One thread a word of eight codes of every gridDim.y-th row.  Where the rows allow it a word's indices are one load of eight bytes
// (28672 x 8192: 90 us, 3.9 TB/s; byte by byte 146).
__global__ void __launch_bounds__(256) k_pack(const uint8_t *__restrict__ idx, int64_t idx_row, int64_t n, int64_t k,
                                              uint8_t *__restrict__ codes, int64_t code_row, int64_t words) {
    const bool vec = ((reinterpret_cast<uintptr_t>(idx) | (uintptr_t)idx_row) & 7) == 0;
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= words) return;
#pragma unroll 4
    for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const uint8_t *from = idx + r * idx_row + 8 * w;
        uint32_t v = 0;
        if (vec && 8 * w + 8 <= k) {
            const uint2 x = *reinterpret_cast<const uint2 *>(from);
            v = four_codes(x.x) | four_codes(x.y) << 16;
        } else {
            for (int j = 0; j < 8; j++)
                if (8 * w + j < k) v |= (uint32_t)(from[j] & 15) << (4 * j);
        }
        const int64_t at = (w & ~(int64_t)15) + packed_word((int)(w & 15));
        *reinterpret_cast<uint32_t *>(codes + r * code_row + 4 * at) = v;
    }
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
    const int64_t across = cdiv(words, 256), down = std::min(n, cdiv(152 * 16, across));
    k_pack<<<dim3((unsigned)across, (unsigned)down), 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(idx, idx_row, n, k, codes, code_row, words);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

int ecasq_matvec(const void *x, int64_t x_row, int32_t type, int64_t b, const uint8_t *codes, int64_t code_row,
                 const void *levels, int32_t m, const void *scales, int64_t scale_row, int32_t scale_type, int64_t n,
                 int64_t k, int32_t group, void *y, int64_t y_row, int32_t *status, ecasq_stream_t stream) {
    const bool lost_wait = (type & ECASQ_TEST_LOST_WAIT) != 0;
    type &= ~ECASQ_TEST_LOST_WAIT;
    if (n < 1 || k < 1 || b < 0 || n >= (int64_t)1 << 31 || k >= (int64_t)1 << 31 || b > 8 * 65535 || m < 1 || m > 16 ||
        !type_ok(type) || (scale_type != type && scale_type != ECASQ_F32) || group < 32 || group % 32)
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!x || !codes || !levels || !scales || !y || !aligned16(codes) || code_row % 16 || code_row < 64 * cdiv(k, 128) ||
        scale_row < cdiv(k, group) || (b > 1 && (x_row < k || y_row < n)))
        return ECASQ_EINVAL;
    MatvecArgs a{};
    a.x = x;
    a.levels = levels;
    a.scales = scales;
    a.codes = codes;
    a.y = y;
    a.status = status;
    a.x_row = x_row;
    a.code_row = code_row;
    a.scale_row = scale_row;
    a.y_row = y_row;
    a.n = n;
    a.k = k;
    a.b = (int32_t)b;
    a.m = m;
    a.groups = (int32_t)cdiv(k, group);
    a.lost = lost_wait;
    const FastDiv div(group / 32);
    a.div_mul = div.mul;
    a.div_shift = div.shift;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (type == ECASQ_F32) return launch_matvec_f32(a, kPlain, group, st);
    return launch_matvec_types<kPlain>(a, type, scale_type == ECASQ_F32, group, st);
}

}  // extern "C"
