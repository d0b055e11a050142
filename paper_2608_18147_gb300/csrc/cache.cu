// cache.cu -- stochastic rounding of new cache rows to 4-bit codes (ecasq_cache_write).
#include <algorithm>

#include "codes.cuh"
#include "draw.cuh"

namespace ecasq {

// Four neighbouring entries; one load where their address allows it.
__device__ __forceinline__ void load4(const float *p, float (&v)[4]) {
    if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        const float4 x = *reinterpret_cast<const float4 *>(p);
        v[0] = x.x;
        v[1] = x.y;
        v[2] = x.z;
        v[3] = x.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) v[j] = p[j];
    }
}
template <typename X> __device__ __forceinline__ void load4(const X *p, float (&v)[4]) {
    alignas(8) X x[4];
    if ((reinterpret_cast<uintptr_t>(p) & 7) == 0) {
        *reinterpret_cast<uint2 *>(x) = *reinterpret_cast<const uint2 *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) x[j] = p[j];
    }
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = to_f32(x[j]);
}

struct WriteArgs {
    const void *x;
    const float *Q;
    const int32_t *m;
    const int64_t *slots;
    ecasq_cache_t c;
    int64_t x_row, x_head, rows;  // rows: n heads
    uint64_t seed;
    int32_t s;
    int32_t *status;
    FastDiv heads, page;          // for row numbers and slots below 2^31
    bool far_rows, far_slots;     // there are others
};

__device__ __forceinline__ int64_t quotient(int64_t v, const FastDiv &f, int32_t n, bool far) {
    if (far) return v / n;
    return f.mul ? __umulhi((uint32_t)v, f.mul) >> f.shift : (uint32_t)v >> f.shift;
}

// LV levels a row.  W lanes take a row, four neighbouring entries at a time each: 8, 16 or 32 for rows of up to 32, 64 or
// more entries.  The row's levels and the gaps above them lie in shared memory, a word a bank, so lanes that look
// up different levels do not meet.
//
// What bounds it: instruction issue, as in the flat encode; the rule's draw alone is about 20 instructions an
// entry.  So the draw is the 32-bit form of draw.cuh, the search takes log2 LV steps, and the gaps are formed once a row;
// an entry equal to its level needs no test (its distance 0 is above no product), nor does one at or beyond the last level
// (the gap there is infinite).
constexpr int kWriteThreads = 256;
template <typename X, typename T, int LV, int W>
__global__ void __launch_bounds__(kWriteThreads) k_cache_write(const __grid_constant__ WriteArgs a) {
    constexpr int kRows = kWriteThreads / W;  // of a block at a time
    __shared__ float books[kRows][32];        // levels, NaN beyond the last (no entry passes it), and gaps from word 16 on
    const int lane = threadIdx.x % W;
    float *book = books[threadIdx.x / W];
    int bad = 0;
    const unsigned mask = W == 32 ? 0xffffffffu : ((1u << W % 32) - 1) << (threadIdx.x % 32 / W * W);
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / W; row < a.rows; row += (int64_t)gridDim.x * kRows) {
        const int64_t i = quotient(row, a.heads, a.c.heads, a.far_rows), h = row - i * a.c.heads, slot = a.slots[i];
        if (slot < 0) continue;
        if (slot >= a.c.pages * a.c.page_size) {  // (before the division, which below 2^31 slots takes 32 bits)
            bad |= ECASQ_BAD_PAGE;
            continue;
        }
        const int64_t page = quotient(slot, a.page, a.c.page_size, a.far_slots);
        const int64_t at = slot - page * a.c.page_size;
        const X *x = static_cast<const X *>(a.x) + i * a.x_row + h * a.x_head;
        int m = a.m ? a.m[row] : a.s;
        if (m < 1 || m > a.s) {
            bad |= ECASQ_BAD_COUNT;
            m = m < 1 ? 1 : a.s;
        }
        __syncwarp(mask);  // the row before is done with the book
#pragma unroll
        for (int j = lane; j < LV; j += W) {
            const float *q = a.Q + row * a.s;
            const T r = from_f32<T>(q[min(j, m - 1)]);
            static_cast<T *>(a.c.levels)[page * a.c.level_page + at * a.c.level_slot + h * a.c.level_head + j] = r;
            const float v = to_f32(r), above = j + 1 < m ? to_f32(from_f32<T>(q[j + 1])) : 0.f;
            book[j] = j < m ? v : CUDART_NAN_F;
            book[16 + j] = j + 1 < m ? __fsub_rn(above, v) : CUDART_INF_F;
        }
        __syncwarp(mask);
        uint8_t *codes = static_cast<uint8_t *>(a.c.rows) + page * a.c.row_page + at * a.c.row_slot + h * a.c.row_head;
        for (int e = 4 * lane; e < a.c.d; e += 4 * W) {
            float v[4];
            load4(x + e, v);
            const uint64_t z = a.seed + (uint64_t)(row * a.c.d + e + 1) * kGamma;
            uint32_t zl = (uint32_t)z, zh = (uint32_t)(z >> 32), word = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (!isfinite(v[j])) bad |= ECASQ_BAD_VALUE;
                int t = 0;
#pragma unroll
                for (int b = LV / 2; b; b >>= 1)
                    if (book[t + b] <= v[j]) t += b;
                const float k = __fmul_rn((float)(splitmix64_hi(zl, zh) >> 8), 0x1p-24f);
                if (__fmul_rn(k, book[16 + t]) < __fsub_rn(v[j], book[t])) t++;
                word |= t << (4 * j);
                add_gamma(zl, zh);
            }
            *reinterpret_cast<uint16_t *>(codes + e / 2) = (uint16_t)word;
        }
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

template <typename X, typename T, int LV>
static void launch_write(const WriteArgs &a, cudaStream_t st) {
    const int w = a.c.d <= 32 ? 8 : a.c.d <= 64 ? 16 : 32;
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv(a.rows, kWriteThreads / w), 152 * 32);
    if (w == 8) k_cache_write<X, T, LV, 8><<<blocks, kWriteThreads, 0, st>>>(a);
    else if (w == 16) k_cache_write<X, T, LV, 16><<<blocks, kWriteThreads, 0, st>>>(a);
    else k_cache_write<X, T, LV, 32><<<blocks, kWriteThreads, 0, st>>>(a);
}
template <typename X, typename T>
static void launch_write(const WriteArgs &a, cudaStream_t st) {
    if (a.c.levels_n == 8) launch_write<X, T, 8>(a, st);
    else launch_write<X, T, 16>(a, st);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

int ecasq_cache_write(const void *x, int32_t x_type, int64_t n, int64_t x_row, int64_t x_head, const float *Q,
                      int32_t s, const int32_t *m, const int64_t *slots, const ecasq_cache_t *cache, uint64_t seed,
                      int32_t *status, ecasq_stream_t stream) {
    if (!cache_ok(cache) || !cache->levels_n || n < 0 || s < 1 || s > cache->levels_n ||
        (x_type != ECASQ_F32 && x_type != cache->type) || n > ((int64_t)1 << 33) / cache->heads)
        return ECASQ_EINVAL;
    if (n == 0) return ECASQ_OK;
    if (!x || !Q || !slots) return ECASQ_EINVAL;
    const int64_t rows = n * cache->heads, near = (int64_t)1 << 31;
    const WriteArgs a{x, Q, m, slots, *cache, x_row, x_head, rows, seed, s, status, FastDiv(cache->heads), FastDiv(cache->page_size),
                      rows >= near, cache->pages * cache->page_size >= near};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    note_launch();
    if (cache->type == ECASQ_F16) {
        if (x_type == ECASQ_F32) launch_write<float, __half>(a, st);
        else launch_write<__half, __half>(a, st);
    } else {
        if (x_type == ECASQ_F32) launch_write<float, __nv_bfloat16>(a, st);
        else launch_write<__nv_bfloat16, __nv_bfloat16>(a, st);
    }
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

}  // extern "C"
