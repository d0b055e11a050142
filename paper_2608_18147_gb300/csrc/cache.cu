// cache.cu -- stochastic rounding of new cache rows to 4-bit codes (ecasq_cache_write).
#include <algorithm>
#include <type_traits>

#include "codes.cuh"
#include "draw.cuh"

namespace ecasq {

// E neighbouring entries as they lie in memory; loads of 8 or 16 bytes where their address allows it.
template <typename X, int E> struct Entries {
    X v[E];
};
template <typename X, int E> __device__ __forceinline__ Entries<X, E> load_entries(const X *p) {
    constexpr int kBytes = E * sizeof(X), kVec = kBytes < 16 ? 8 : 16;
    using Vec = std::conditional_t<kVec == 8, uint2, uint4>;
    alignas(16) Entries<X, E> x;
    if ((reinterpret_cast<uintptr_t>(p) & (kVec - 1)) == 0) {
#pragma unroll
        for (int i = 0; i < kBytes / kVec; i++) reinterpret_cast<Vec *>(x.v)[i] = reinterpret_cast<const Vec *>(p)[i];
    } else {
#pragma unroll
        for (int j = 0; j < E; j++) x.v[j] = p[j];
    }
    return x;
}

// I: row numbers, slots and strides, 32 bits where all of them are below 2^31 (8191 x 8 rows of 128: 19.8 us, and 22.8 in 64 bits).
template <typename I> struct WriteArgs {
    const void *x;
    const float *Q;
    const int32_t *m;
    const int64_t *slots;
    uint8_t *codes;
    void *levels;
    int64_t end;                  // slots of the cache
    uint64_t seed;
    int32_t *status;
    I x_row, x_head, row_page, row_slot, row_head, level_page, level_slot, level_head, rows;  // strides as in ecasq_cache_t; rows: n heads
    int32_t s, d, heads, page_size;
    FastDiv by_heads, by_page;
};

template <typename I> __device__ __forceinline__ I quotient(I v, const FastDiv &f, int32_t n) {
    if (sizeof(I) == 8) return v / n;
    return f.mul ? __umulhi((uint32_t)v, f.mul) >> f.shift : (uint32_t)v >> f.shift;
}
__device__ __forceinline__ uint64_t product(uint32_t a, uint32_t b) { return (uint64_t)a * b; }
__device__ __forceinline__ int64_t product(int64_t a, int64_t b) { return a * b; }
// The largest finite value of a 16-bit type, as its bits, and the least fp32 that rounds beyond it.
template <typename T> struct Range;
template <> struct Range<__half> {
    static constexpr uint16_t kMost = 0x7BFF;
    static constexpr float kBeyond = 65520.f;
};
template <> struct Range<__nv_bfloat16> {
    static constexpr uint16_t kMost = 0x7F7F;
    static constexpr float kBeyond = 0x1.FFp127f;
};
__device__ __forceinline__ float shared_float(uint32_t at) { return *static_cast<const float *>(__cvta_shared_to_generic(at)); }

// LV levels a row.  W lanes take a row, E neighbouring entries each: 16 lanes with four for rows of up to 64 entries, with eight
// for up to 128, 32 lanes with eight for the others (a row's own cost, addresses and levels, is shared by more entries, and no
// lane rests: 8191 x 8 rows of 128 take 19.4 us, and 36.8 with 32 lanes a row; rows of 64 12.8 us, and 19.4 with eight entries a lane).
// The row's levels and the gaps above them lie in shared memory, a word a bank, so lanes that look up different levels
// do not meet.
//
// What bounds it: instruction issue (71 % of the slots, 62 instructions an entry), as in the flat encode; 8191 x 8 rows of 128
// take 19.1 us, 1.4 TB/s or 440 entries a nanosecond, a step of 32 x 8 rows 2.4 us.  The rule's draw alone is about 20 instructions an
// entry.  So the draw is the 32-bit form of draw.cuh, the search takes log2 LV steps, and the gaps are formed once a row;
// an entry equal to its level needs no test (its distance 0 is above no product), nor does one at or beyond the last level
// (the gap there is infinite).  The search's position is a shared-memory address that steps by predicated fp32 additions of
// its bits, denormals whose sums are exact, on the pipe that has room.  The next row is on its way while this one is
// encoded.
constexpr int kWriteThreads = 256;
template <typename X, typename T, int LV, int W, int E, typename I>
__global__ void __launch_bounds__(kWriteThreads) k_cache_write(const __grid_constant__ WriteArgs<I> a) {
    constexpr int kRows = kWriteThreads / W;  // of a block at a time
    __shared__ float books[kRows][48];        // levels, NaN beyond the last (no entry passes it), and gaps from word 16 on; two
                                              // rows of a warp do not meet in a bank
    const int lane = threadIdx.x % W;
    float *book = books[threadIdx.x / W];
    const uint32_t book_at = (uint32_t)__cvta_generic_to_shared(book);
    const unsigned group = W == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);  // the row's lanes
    struct Row {
        int64_t slot;
        I i, h;
        int m;
        float q;
        Entries<X, E> x;
    };
    auto row_of_x = [&](I i, I h) { return static_cast<const X *>(a.x) + product(i, a.x_row) + product(h, a.x_head); };
    auto fetch = [&](I row) {
        Row r;
        r.i = quotient(row, a.by_heads, a.heads);
        r.h = row - r.i * (I)a.heads;
        r.slot = a.slots[r.i];
        r.m = a.m ? a.m[row] : a.s;
        r.q = lane < a.s ? a.Q[product(row, (I)a.s) + lane] : 0.f;
        if (E * lane < a.d) r.x = load_entries<X, E>(row_of_x(r.i, r.h) + E * lane);
        return r;
    };
    wait_before();
    int bad = 0;
    const I stride = (I)gridDim.x * kRows;
    I row = (I)blockIdx.x * kRows + threadIdx.x / W;
    Row next;
    if (row < a.rows) next = fetch(row);
    for (; row < a.rows; row += stride) {
        const Row r = next;
        if (a.rows - row > stride) next = fetch(row + stride);
        if (r.slot < 0) continue;
        if (r.slot >= a.end) {  // (before the division, which below 2^31 slots takes 32 bits)
            bad |= ECASQ_BAD_PAGE;
            continue;
        }
        const I page = quotient((I)r.slot, a.by_page, a.page_size), at = (I)r.slot - page * (I)a.page_size;
        const int m = min(max(r.m, 1), a.s);
        if (m != r.m) bad |= ECASQ_BAD_COUNT;
        __syncwarp(group);  // the row before is done with the book
        T rounded = from_f32<T>(r.q);  // (a comparison and a choice; a rounding that saturates took 0.2 us more for 8191 x 8 rows of 64)
        if (lane < m && !(fabsf(r.q) < Range<T>::kBeyond)) {
            bad |= ECASQ_BAD_VALUE;
            const uint16_t most = Range<T>::kMost | (uint16_t)(__float_as_uint(r.q) >> 16 & 0x8000u);
            if (r.q == r.q) rounded = reinterpret_cast<const T &>(most);
        }
        const float mine = to_f32(rounded), last = __shfl_sync(group, mine, m - 1, W), above = __shfl_down_sync(group, mine, 1, W);
        if (lane < LV) {
            T *levels = static_cast<T *>(a.levels) + product(page, a.level_page) + product(at, a.level_slot) + product(r.h, a.level_head);
            levels[lane] = lane < m ? rounded : from_f32<T>(last);
            book[lane] = lane < m ? mine : CUDART_NAN_F;
            book[16 + lane] = lane + 1 < m ? __fsub_rn(above, mine) : CUDART_INF_F;
        }
        __syncwarp(group);
        uint8_t *codes = a.codes + product(page, a.row_page) + product(at, a.row_slot) + product(r.h, a.row_head);
        if (E * lane < a.d) {
            const uint64_t z = a.seed + ((uint64_t)row * (uint32_t)a.d + E * lane + 1) * kGamma;
            uint32_t zl = (uint32_t)z, zh = (uint32_t)(z >> 32), word = 0;
            float largest = 0.f;
#pragma unroll
            for (int j = 0; j < E; j++) {
                const float v = to_f32(r.x.v[j]);
                asm("max.NaN.f32 %0, %0, %1;" : "+f"(largest) : "f"(fabsf(v)));
                float t = __uint_as_float(book_at);  // the address of the largest level passed
#pragma unroll
                for (int b = LV / 2; b; b >>= 1)
                    if (shared_float(__float_as_uint(t) + 4 * b) <= v) t = __fadd_rn(t, __uint_as_float(4 * b));
                const float k = __fmul_rn((float)(splitmix64_hi(zl, zh) >> 8), 0x1p-24f);
                if (__fmul_rn(k, shared_float(__float_as_uint(t) + 64)) < __fsub_rn(v, shared_float(__float_as_uint(t))))
                    t = __fadd_rn(t, __uint_as_float(4));
                word += ((__float_as_uint(t) - book_at) >> 2) << (4 * j);
                add_gamma(zl, zh);
            }
            if (!(largest <= 3.402823466e38f)) bad |= ECASQ_BAD_VALUE;
            if (E == 8) reinterpret_cast<uint32_t *>(codes)[lane] = word;
            else reinterpret_cast<uint16_t *>(codes)[lane] = (uint16_t)word;
        }
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

template <typename X, typename T, typename I>
static int launch_write(const WriteArgs<I> &a, int32_t levels, cudaStream_t st) {
    const int lanes = a.d <= 128 ? 16 : 32;
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv((int64_t)a.rows, kWriteThreads / lanes), 152 * 8);
    auto *kernel = levels == 8 ? (a.d <= 64 ? k_cache_write<X, T, 8, 16, 4, I> : a.d <= 128 ? k_cache_write<X, T, 8, 16, 8, I> : k_cache_write<X, T, 8, 32, 8, I>)
                               : (a.d <= 64 ? k_cache_write<X, T, 16, 16, 4, I> : a.d <= 128 ? k_cache_write<X, T, 16, 16, 8, I> : k_cache_write<X, T, 16, 32, 8, I>);
    return launch_early(kernel, dim3(blocks), kWriteThreads, 0, st, a);
}
template <typename I>
static int write_rows(const void *x, int32_t x_type, int64_t n, int64_t x_row, int64_t x_head, const float *Q, int32_t s, const int32_t *m,
                      const int64_t *slots, const ecasq_cache_t &c, uint64_t seed, int32_t *status, cudaStream_t st) {
    const WriteArgs<I> a{x, Q, m, slots, static_cast<uint8_t *>(c.rows), c.levels, c.pages * c.page_size, seed, status, (I)x_row, (I)x_head,
                         (I)c.row_page, (I)c.row_slot, (I)c.row_head, (I)c.level_page, (I)c.level_slot, (I)c.level_head,
                         (I)(n * c.heads), s, c.d, c.heads, c.page_size, FastDiv(c.heads), FastDiv(c.page_size)};
    if (c.type == ECASQ_F16) return x_type == ECASQ_F32 ? launch_write<float, __half>(a, c.levels_n, st) : launch_write<__half, __half>(a, c.levels_n, st);
    return x_type == ECASQ_F32 ? launch_write<float, __nv_bfloat16>(a, c.levels_n, st) : launch_write<__nv_bfloat16, __nv_bfloat16>(a, c.levels_n, st);
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
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const ecasq_cache_t &c = *cache;
    bool near = true;
    for (const int64_t v : {x_row, x_head, c.row_page, c.row_slot, c.row_head, c.level_page, c.level_slot, c.level_head, n * c.heads,
                            c.pages * c.page_size})
        near = near && v >= 0 && v < (int64_t)1 << 31;
    return near ? write_rows<uint32_t>(x, x_type, n, x_row, x_head, Q, s, m, slots, c, seed, status, st)
                : write_rows<int64_t>(x, x_type, n, x_row, x_head, Q, s, m, slots, c, seed, status, st);
}

}  // extern "C"
