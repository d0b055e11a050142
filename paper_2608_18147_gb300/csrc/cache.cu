// cache.cu -- stochastic rounding of new cache rows to 4-bit codes (ecasq_cache_write).
#include <algorithm>

#include "codes.cuh"

namespace ecasq {

constexpr uint64_t kCounterStep = 0x9E3779B97F4A7C15ull;  // SplitMix64 (Steele, Lea and Flood 2014)

__device__ __forceinline__ uint32_t draw24(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return (uint32_t)(z >> 40);  // the last xor-shift leaves the top 31 bits as they are
}

struct WriteArgs {
    const void *x;
    const float *Q;
    const int32_t *m;
    const int64_t *slots;
    ecasq_cache_t c;
    int64_t x_row, x_head, n;
    uint64_t seed;
    int32_t s;
    int32_t *status;
};

// One warp a row, each lane every 32nd pair of entries.
template <typename X, typename T>
__global__ void __launch_bounds__(256) k_cache_write(WriteArgs a) {
    __shared__ float book[8][16];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * 8 + wid;
    if (row >= a.n * a.c.heads) return;
    const int64_t i = row / a.c.heads, h = row % a.c.heads, slot = a.slots[i];
    if (slot < 0) return;
    int bad = 0;
    if (slot >= a.c.pages * a.c.page_size) {
        if (lane == 0 && a.status) atomicOr(a.status, ECASQ_BAD_PAGE);
        return;
    }
    int m = a.m ? a.m[row] : a.s;
    if (m < 1 || m > a.s) {
        bad |= ECASQ_BAD_COUNT;
        m = m < 1 ? 1 : a.s;
    }
    const int64_t page = slot / a.c.page_size, at = slot % a.c.page_size;
    uint8_t *codes = static_cast<uint8_t *>(a.c.rows) + page * a.c.row_page + at * a.c.row_slot + h * a.c.row_head;
    T *levels = static_cast<T *>(a.c.levels) + page * a.c.level_page + at * a.c.level_slot + h * a.c.level_head;
    if (lane < a.c.levels_n) {
        const T r = from_f32<T>(a.Q[row * a.s + min(lane, m - 1)]);
        levels[lane] = r;
        book[wid][lane] = to_f32(r);
    }
    __syncwarp();
    const float *q = book[wid];
    const X *x = static_cast<const X *>(a.x) + i * a.x_row + h * a.x_head;
    for (int e = 2 * lane; e < a.c.d; e += 64) {
        int byte = 0;
        for (int j = 0; j < 2; j++) {
            const float v = to_f32(x[e + j]);
            if (!isfinite(v)) bad |= ECASQ_BAD_VALUE;
            int t = 0;
            for (int u = 1; u < m; u++)
                if (q[u] <= v) t = u;
            if (t < m - 1 && q[t] != v) {
                const uint64_t z = a.seed + (uint64_t)(row * a.c.d + e + j + 1) * kCounterStep;
                const float kf = __fmul_rn((float)draw24(z), 0x1p-24f);
                if (__fmul_rn(kf, __fsub_rn(q[t + 1], q[t])) < __fsub_rn(v, q[t])) t++;
            }
            byte |= t << (4 * j);
        }
        codes[e / 2] = (uint8_t)byte;
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

template <typename X, typename T>
static void launch_write(const WriteArgs &a, cudaStream_t st) {
    k_cache_write<X, T><<<(unsigned)cdiv(a.n * a.c.heads, 8), 256, 0, st>>>(a);
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
    const WriteArgs a{x, Q, m, slots, *cache, x_row, x_head, n, seed, s, status};
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
