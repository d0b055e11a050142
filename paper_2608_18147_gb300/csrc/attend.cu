// attend.cu -- attention of one new token a sequence over a paged cache (ecasq_attend).
#include <algorithm>

#include "codes.cuh"

namespace ecasq {

struct AttendArgs {
    const void *q;
    void *out;
    const int32_t *table, *lengths, *starts;
    float *lse;
    int32_t *status;
    ecasq_cache_t k, v;
    int64_t q_row, q_head, out_row, out_head, table_row, max_len;
    float scale;
    int heads;
};

template <typename T>
__device__ __forceinline__ float entry(const ecasq_cache_t &c, int64_t page, int64_t slot, int64_t head, int e) {
    if (!c.levels_n) return to_f32(static_cast<const T *>(c.rows)[page * c.row_page + slot * c.row_slot + head * c.row_head + e]);
    const uint8_t byte = static_cast<const uint8_t *>(c.rows)[page * c.row_page + slot * c.row_slot + head * c.row_head + e / 2];
    const T *levels = static_cast<const T *>(c.levels) + page * c.level_page + slot * c.level_slot + head * c.level_head;
    return to_f32(levels[(e & 1 ? byte >> 4 : byte & 15) & (c.levels_n - 1)]);
}

// One block a sequence and query head, 128 keys at a time: a thread a key for the scores, a
// thread two entries for the sums.
template <typename T>
__global__ void __launch_bounds__(128) k_attend(AttendArgs a) {
    __shared__ float q[256], p[128], red[4];
    __shared__ int64_t pages[128];
    const int64_t seq = blockIdx.y;
    const int h = blockIdx.x, d = a.k.d, kh = h / (a.heads / a.k.heads), tid = threadIdx.x;
    for (int e = tid; e < d; e += 128) q[e] = to_f32(static_cast<const T *>(a.q)[seq * a.q_row + h * a.q_head + e]);
    int64_t end = a.lengths[seq], first = a.starts ? max(0, a.starts[seq]) : 0;
    int bad = 0;
    if (end > a.max_len) { end = a.max_len; bad = ECASQ_BAD_LENGTH; }
    float top = -CUDART_INF_F, total = 0.f, acc[2] = {0.f, 0.f};
    for (int64_t t0 = first; t0 < end; t0 += 128) {
        const int64_t t = t0 + tid;
        float s = -CUDART_INF_F;
        __syncthreads();
        pages[tid] = -1;
        if (t < end) {
            const int64_t page = a.table[seq * a.table_row + t / a.k.page_size];
            if (page < 0 || page >= a.k.pages) bad |= ECASQ_BAD_PAGE;
            else {
                pages[tid] = page;
                s = 0.f;
                for (int e = 0; e < d; e++) s = fmaf(q[e], entry<T>(a.k, page, t % a.k.page_size, kh, e), s);
                s *= a.scale;
            }
        }
        float mx = s;
        for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if ((tid & 31) == 0) red[tid >> 5] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), top);
        const float base = mx == -CUDART_INF_F ? 0.f : mx, shrink = expf(top - base);
        p[tid] = expf(s - base);
        __syncthreads();
        total *= shrink;
        acc[0] *= shrink;
        acc[1] *= shrink;
        top = mx;
        for (int j = 0; j < 128 && t0 + j < end; j++) {
            if (pages[j] < 0) continue;
            total += p[j];
            for (int u = 0; u < 2; u++)
                if (tid + 128 * u < d)
                    acc[u] = fmaf(p[j], entry<T>(a.v, pages[j], (t0 + j) % a.k.page_size, kh, tid + 128 * u), acc[u]);
        }
    }
    for (int u = 0; u < 2; u++)
        if (tid + 128 * u < d)
            static_cast<T *>(a.out)[seq * a.out_row + h * a.out_head + tid + 128 * u] =
                from_f32<T>(total == 0.f ? 0.f : acc[u] / total);
    if (tid == 0 && a.lse) a.lse[seq * a.heads + h] = total == 0.f ? -CUDART_INF_F : top + logf(total);
    if (bad && a.status) atomicOr(a.status, bad);
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

size_t ecasq_workspace_size_attend(int64_t b, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_len) {
    return 0;
}

int ecasq_attend(const void *q, int64_t q_row, int64_t q_head, int64_t b, int32_t heads, const ecasq_cache_t *k,
                 const ecasq_cache_t *v, const int32_t *table, int64_t table_row, const int32_t *lengths,
                 const int32_t *starts, int64_t max_len, float scale, void *out, int64_t out_row, int64_t out_head,
                 float *lse, void *ws, size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    if (!cache_ok(k) || !cache_ok(v) || k->type != v->type || k->levels_n != v->levels_n || k->d != v->d ||
        k->heads != v->heads || k->pages != v->pages || k->page_size != v->page_size || b < 0 || b > 65535 || heads < 1 ||
        heads % k->heads || max_len < 0 || max_len >= (int64_t)1 << 31)
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!q || !out || !lengths || (max_len && (!table || table_row < cdiv(max_len, k->page_size)))) return ECASQ_EINVAL;
    const AttendArgs a{q, out, table, lengths, starts, lse, status, *k, *v, q_row, q_head, out_row, out_head,
                       table_row, max_len, scale, heads};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)heads, (unsigned)b);
    note_launch();
    if (k->type == ECASQ_F32) k_attend<float><<<grid, 128, 0, st>>>(a);
    else if (k->type == ECASQ_F16) k_attend<__half><<<grid, 128, 0, st>>>(a);
    else k_attend<__nv_bfloat16><<<grid, 128, 0, st>>>(a);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

}  // extern "C"
