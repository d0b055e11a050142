// cache.cu -- stochastic rounding of new cache rows to 4-bit codes (ecasq_cache_write).
#include <algorithm>
#include <type_traits>

#include "codes.cuh"
#include "draw.cuh"

namespace ecasq {

// Four neighbouring entries as they lie in memory; one load where their address allows it.
template <typename X> struct Four {
    X v[4];
};
template <typename X> __device__ __forceinline__ Four<X> load4(const X *p) {
    using Vec = std::conditional_t<sizeof(X) == 4, uint4, uint2>;
    alignas(16) Four<X> x;
    if ((reinterpret_cast<uintptr_t>(p) & (sizeof(Vec) - 1)) == 0) {
        *reinterpret_cast<Vec *>(x.v) = *reinterpret_cast<const Vec *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) x.v[j] = p[j];
    }
    return x;
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
    FastDiv heads, page;
};

// LV levels a row.  W lanes take a row, four neighbouring entries at a time each: 16 for rows of up to 64 entries, else 32.
// The row's levels and the gaps above them lie in shared memory, a word a bank, so lanes that look up different levels
// do not meet.  I: row numbers and slots, 32 bits where they are below 2^31.
//
// What bounds it: instruction issue, as in the flat encode; the rule's draw alone is about 20 instructions an
// entry.  So the draw is the 32-bit form of draw.cuh, the search takes log2 LV steps, and the gaps are formed once a row;
// an entry equal to its level needs no test (its distance 0 is above no product), nor does one at or beyond the last level
// (the gap there is infinite).  The next row is on its way while this one is encoded.
constexpr int kWriteThreads = 256;
template <typename X, typename T, int LV, int W, typename I>
__global__ void __launch_bounds__(kWriteThreads) k_cache_write(const __grid_constant__ WriteArgs a) {
    constexpr int kRows = kWriteThreads / W;  // of a block at a time
    __shared__ float books[kRows][32];        // levels, NaN beyond the last (no entry passes it), and gaps from word 16 on
    const int lane = threadIdx.x % W;
    float *book = books[threadIdx.x / W];
    const unsigned group = W == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);  // the row's lanes
    auto quotient = [](I v, const FastDiv &f, int32_t n) -> I {
        if (sizeof(I) == 8) return v / n;
        return f.mul ? __umulhi((uint32_t)v, f.mul) >> f.shift : (uint32_t)v >> f.shift;
    };
    struct Row {
        int64_t slot;
        I i, h;
        int m;
        float q;
        Four<X> x;
    };
    auto fetch = [&](I row) {
        Row r;
        r.i = quotient(row, a.heads, a.c.heads);
        r.h = row - r.i * (I)a.c.heads;
        r.slot = a.slots[r.i];
        r.m = a.m ? a.m[row] : a.s;
        r.q = lane < a.s ? a.Q[(int64_t)row * a.s + lane] : 0.f;
        if (4 * lane < a.c.d) r.x = load4(static_cast<const X *>(a.x) + (int64_t)r.i * a.x_row + (int64_t)r.h * a.x_head + 4 * lane);
        return r;
    };
    int bad = 0;
    const I stride = (I)gridDim.x * kRows;
    I row = (I)blockIdx.x * kRows + threadIdx.x / W;
    Row next;
    if (row < (I)a.rows) next = fetch(row);
    for (; row < (I)a.rows; row += stride) {
        const Row r = next;
        if ((I)a.rows - row > stride) next = fetch(row + stride);
        if (r.slot < 0) continue;
        if (r.slot >= a.c.pages * a.c.page_size) {  // (before the division, which below 2^31 slots takes 32 bits)
            bad |= ECASQ_BAD_PAGE;
            continue;
        }
        const I page = quotient((I)r.slot, a.page, a.c.page_size), at = (I)r.slot - page * (I)a.c.page_size;
        const int m = min(max(r.m, 1), a.s);
        if (m != r.m) bad |= ECASQ_BAD_COUNT;
        __syncwarp(group);  // the row before is done with the book
        const T rounded = from_f32<T>(r.q);
        const float mine = to_f32(rounded), last = __shfl_sync(group, mine, m - 1, W), above = __shfl_down_sync(group, mine, 1, W);
        if (lane < LV) {
            T *levels = static_cast<T *>(a.c.levels) + ((int64_t)page * a.c.level_page + (int64_t)at * a.c.level_slot + (int64_t)r.h * a.c.level_head);
            levels[lane] = lane < m ? rounded : from_f32<T>(last);
            book[lane] = lane < m ? mine : CUDART_NAN_F;
            book[16 + lane] = lane + 1 < m ? __fsub_rn(above, mine) : CUDART_INF_F;
        }
        __syncwarp(group);
        uint8_t *codes = static_cast<uint8_t *>(a.c.rows) + ((int64_t)page * a.c.row_page + (int64_t)at * a.c.row_slot + (int64_t)r.h * a.c.row_head);
        Four<X> x = r.x;
        uint64_t z = a.seed + ((uint64_t)row * (uint32_t)a.c.d + 4 * lane + 1) * kGamma;
        for (int e = 4 * lane; e < a.c.d; e += 4 * W) {
            uint32_t zl = (uint32_t)z, zh = (uint32_t)(z >> 32), word = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float v = to_f32(x.v[j]);
                if (!isfinite(v)) bad |= ECASQ_BAD_VALUE;
                int t = 0;
#pragma unroll
                for (int b = LV / 2; b; b >>= 1)
                    if (book[t + b] <= v) t += b;
                const float k = __fmul_rn((float)(splitmix64_hi(zl, zh) >> 8), 0x1p-24f);
                if (__fmul_rn(k, book[16 + t]) < __fsub_rn(v, book[t])) t++;
                word |= t << (4 * j);
                add_gamma(zl, zh);
            }
            *reinterpret_cast<uint16_t *>(codes + e / 2) = (uint16_t)word;
            if (e + 4 * W < a.c.d) x = load4(static_cast<const X *>(a.x) + (int64_t)r.i * a.x_row + (int64_t)r.h * a.x_head + e + 4 * W);
            z += 4 * W * kGamma;
        }
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

template <typename X, typename T, int LV, int W>
static void launch_write_lanes(const WriteArgs &a, cudaStream_t st) {
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv(a.rows, kWriteThreads / W), 152 * 8);
    const int64_t near = ((int64_t)1 << 31) - 1;
    if (a.rows <= near && a.c.pages <= near / a.c.page_size) k_cache_write<X, T, LV, W, uint32_t><<<blocks, kWriteThreads, 0, st>>>(a);
    else k_cache_write<X, T, LV, W, int64_t><<<blocks, kWriteThreads, 0, st>>>(a);
}
template <typename X, typename T, int LV>
static void launch_write(const WriteArgs &a, cudaStream_t st) {
    if (a.c.d <= 64) launch_write_lanes<X, T, LV, 16>(a, st);
    else launch_write_lanes<X, T, LV, 32>(a, st);
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
    const WriteArgs a{x, Q, m, slots, *cache, x_row, x_head, n * cache->heads, seed, s, status, FastDiv(cache->heads), FastDiv(cache->page_size)};
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
