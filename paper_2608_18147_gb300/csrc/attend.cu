// attend.cu -- ecasq_attend: checks, splits and the join of the splits' results.
#include <algorithm>

#include "attend.cuh"

namespace ecasq {

// Splits.  A block has a fixed cost of its own, about what kCost keys take it (its first loads' latency), and the join's launch
// about what kJoinCost keys take, so a split should be long; and the blocks should fill the card evenly: with `slots` of them at
// once, n splits a sequence take ceil(b blocks n / slots) rounds of a split's keys and that cost.  With one round a shorter
// sequence takes shorter splits, so that all blocks still work; with several the splits keep their length, and their number adapts.
constexpr int kSms = 152, kMostResident = 8, kMostRounds = 8, kCost = 96, kLeastStep = 64, kMostTile = 32;
constexpr int kClusterMost = 8, kClusterChunk = 1024, kJoinCost = 64;

// Whether the splits of a sequence are a cluster of blocks that joins them itself, through its shared memory, which saves the join's
// launch.  Clusters do not fill the SMs evenly, larger ones less so, which costs in proportion to a split's keys; so only where
// splits are short and blocks few.  (Eight key heads, four heads each, bf16 keys of 128, by clusters and by the join: one sequence of
// 1000 keys, a head each, 6.0 and 6.5 us, 8 of 600 7.7 and 9.4, 16 of 2000 in three splits 24.9 and 28.0; but 8 of 2000 in
// seven splits, 448 blocks, 23.4 and 18.5, and 32 of up to 8192, eight heads each, 118 and 94.)
static bool by_cluster(int64_t count, int64_t chunk, int64_t blocks, int64_t slots) {
    return count > 1 && count <= kClusterMost && chunk <= kClusterChunk && 2 * blocks <= (count <= kClusterMost / 2 ? 2 * slots : 5 * kSms);
}

struct Splits {
    int32_t least, count;
    bool cluster;
};
static Splits make_splits(int64_t b, int64_t blocks, int64_t span, int64_t slots, int64_t step) {
    const int64_t all = std::max<int64_t>(1, b * blocks);
    Splits best{0, 0, false};
    int64_t least = INT64_MAX;
    const auto consider = [&](int64_t n) {
        const int64_t chunk = std::max<int64_t>(1, cdiv(cdiv(span, n), step)) * step, count = std::max<int64_t>(1, cdiv(span, chunk));
        const bool cluster = by_cluster(count, chunk, all * count, slots);
        const int64_t cost = cdiv(all * count, slots) * (chunk + kCost) + (count > 1 && !cluster ? kJoinCost : 0);
        if (cost < least) {
            least = cost;
            best = {(int32_t)(all * count <= slots ? step : chunk), (int32_t)count, cluster};
        }
        return chunk > step;
    };
    for (int64_t rounds = 1; rounds <= kMostRounds; rounds++) {  // the most splits that this many rounds hold
        const int64_t n = std::max<int64_t>(1, slots * rounds / all);
        if (n > kClusterMost) consider(kClusterMost);
        if (!consider(n)) break;
    }
    return best;
}
// Bytes of the splits' results: room for the most splits that make_splits may choose with as many sequences or with fewer, with
// keys and heads likewise, so that a workspace made for the largest sizes serves all smaller ones.  Where a sequence
// has several splits its blocks are b kv_heads ceil(group / kHeads) and all splits together no more than kMostParts blocks, each with a result for
// min(group, kHeads) heads at most; and a sequence has no more splits than its keys fill.  (Splits count from the tile
// of the first key, so with a start one more tile may be needed.)
constexpr int64_t kMostParts = (int64_t)kSms * kMostResident * kMostRounds;
static size_t part_bytes(int64_t b, int64_t heads, int64_t kv_heads, int32_t d, int64_t max_len) {
    const int64_t splits = cdiv(max_len + kMostTile - 1, kLeastStep);
    return splits > 1 ? (size_t)(std::min(b * heads * splits, kMostParts * std::min<int64_t>(heads / kv_heads, kHeads)) * PartAt(d).stride) * 4 : 0;
}

int split_attend(AttendArgs &a, int64_t b, int resident) {
    const int64_t blocks = (int64_t)(a.heads / a.group) * a.htiles;
    const Splits s = make_splits(b, blocks, a.max_len + (a.starts ? a.tile - 1 : 0), kSms * std::min(resident, kMostResident), a.step);
    a.least = s.least;
    a.splits = s.count;
    a.cluster = s.cluster;
    if (a.splits == 1) return ECASQ_OK;
    if (!a.ws || (reinterpret_cast<uintptr_t>(a.ws) & 255) || a.ws_bytes < part_bytes(b, a.heads, a.heads / a.group, a.d, a.max_len)) return ECASQ_EWORKSPACE;
    a.part = static_cast<float *>(a.ws);
    return ECASQ_OK;
}

// The splits' maxima and sums give each split's share, then the entries are added, four a lane.  A head by a warp (WARPS = 1,
// eight heads a block, nothing to wait for), or 64 entries of a head by a block, 16 splits at a time.  Bound by the latency of
// its loads: 2 to 3 us after the splits' kernel, whose end its start overlaps.
// A sequence of one split has its result already.
constexpr int kJoinThreads = 256, kJoinResident = 4, kShares = 1024;  // kJoinResident: blocks an SM holds
template <typename T, int WARPS>
__global__ void __launch_bounds__(kJoinThreads, kJoinResident) k_attend_join(const __grid_constant__ AttendArgs a) {
    constexpr int kThreads = 32 * WARPS, kHeadsHere = kJoinThreads / kThreads;
    __shared__ float red[2 * WARPS], share[WARPS == 1 ? 1 : kShares];
    __shared__ __align__(16) float4 sums[WARPS == 1 ? 1 : kJoinThreads];
    wait_before();
    const int64_t seq = blockIdx.y;
    const int h = blockIdx.x * kHeadsHere + threadIdx.x / kThreads, tid = threadIdx.x % kThreads, lane = tid & 31, wid = tid >> 5;
    const int n = cut_of(a, seq_span(a, seq)).count;
    const PartAt at(a.d);
    const float *part = at.at(a.part, seq, a.heads, h, a.splits, 0);
    if (n <= 1 || h >= a.heads) return;
    float m = -CUDART_INF_F;
    for (int i = tid; i < n; i += kThreads) m = fmaxf(m, part[i * at.stride + a.d]);
    for (int x = 16; x; x /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    if (WARPS > 1) {
        if (lane == 0) red[wid] = m;
        __syncthreads();
        m = red[0];
        for (int w = 1; w < WARPS; w++) m = fmaxf(m, red[w]);
    }
    const float base = m == -CUDART_INF_F ? 0.f : m;
    float l = 0.f;
    if constexpr (WARPS == 1) {
        const int quads = a.d / 4;
        float4 v[2] = {};  // entries 4 lane .. and 128 + 4 lane ..
        for (int i0 = 0; i0 < n; i0 += 32) {
            float mine = 0.f;
            if (i0 + lane < n) {
                const float2 ml = *reinterpret_cast<const float2 *>(part + (i0 + lane) * at.stride + a.d);
                mine = exp2_fast(ml.x - base);
                l += ml.y * mine;
            }
            const int some = min(32, n - i0);
#pragma unroll 4
            for (int i = 0; i < some; i++) {
                const float s = __shfl_sync(0xffffffffu, mine, i);
#pragma unroll
                for (int c = 0; c < 2; c++)
                    if (lane + 32 * c < quads) {
                        const float4 x = *reinterpret_cast<const float4 *>(part + (i0 + i) * at.stride + 4 * (lane + 32 * c));
                        v[c].x = fmaf(x.x, s, v[c].x);
                        v[c].y = fmaf(x.y, s, v[c].y);
                        v[c].z = fmaf(x.z, s, v[c].z);
                        v[c].w = fmaf(x.w, s, v[c].w);
                    }
            }
        }
        for (int x = 16; x; x /= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
#pragma unroll
        for (int c = 0; c < 2; c++)
            if (lane + 32 * c < quads) store_out<T>(a, seq, h, 4 * (lane + 32 * c), v[c], l);
    } else {
        constexpr int lanes = 16;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        const int e = 64 * blockIdx.z + 4 * (tid % lanes), from = tid / lanes, apart = kThreads / lanes;
        for (int i0 = 0; i0 < n; i0 += kShares) {
            const int some = min(kShares, n - i0);
            const float *p = part + i0 * at.stride;
            for (int i = tid; i < some; i += kThreads) {
                const float2 ml = *reinterpret_cast<const float2 *>(p + i * at.stride + a.d);
                share[i] = exp2_fast(ml.x - base);
                l += ml.y * share[i];
            }
            __syncthreads();
            if (e < a.d) {
#pragma unroll 8
                for (int i = from; i < some; i += apart) {
                    const float4 x = *reinterpret_cast<const float4 *>(p + i * at.stride + e);
                    const float s = share[i];
                    v.x = fmaf(x.x, s, v.x);
                    v.y = fmaf(x.y, s, v.y);
                    v.z = fmaf(x.z, s, v.z);
                    v.w = fmaf(x.w, s, v.w);
                }
            }
            __syncthreads();
        }
        for (int x = 16; x; x /= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
        if (lane == 0) red[WARPS + wid] = l;
        sums[tid] = v;
        __syncthreads();
        l = 0.f;
        for (int w = 0; w < WARPS; w++) l += red[WARPS + w];
        if (tid < lanes && e < a.d) {
            for (int i = 1; i < apart; i++) {
                const float4 x = sums[i * lanes + tid];
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
            }
            store_out<T>(a, seq, h, e, v, l);
        }
    }
    if (tid == 0 && blockIdx.z == 0 && a.lse) a.lse[seq * a.heads + h] = log_sum(m, l);
}

template <typename T>
static int launch_join(const AttendArgs &a, int64_t b, cudaStream_t st) {
    // By warps where blocks would not all run at once.  (32 sequences of 4096 keys, 32 heads of 128: 87.6 us by warps, 94.0 by
    // blocks; one sequence of 2000: 10.6 by warps, 7.2 by blocks.)
    const bool warps = a.heads * b * cdiv(a.d, 64) > kJoinResident * kSms;
    const dim3 grid((unsigned)(warps ? cdiv(a.heads, kJoinThreads / 32) : a.heads), (unsigned)b, (unsigned)(warps ? 1 : cdiv(a.d, 64)));
    return warps ? launch_early(k_attend_join<T, 1>, grid, kJoinThreads, 0, st, a) : launch_early(k_attend_join<T, kJoinThreads / 32>, grid, kJoinThreads, 0, st, a);
}

static bool sizes_ok(int64_t b, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_len) {
    return b >= 0 && b <= 65535 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && heads <= 65535 && d >= 1 && d <= 256 && max_len >= 0 &&
           max_len <= (int64_t)1 << 30;
}

}  // namespace ecasq

using namespace ecasq;

extern "C" {

size_t ecasq_workspace_size_attend(int64_t b, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_len) {
    if (!sizes_ok(b, heads, kv_heads, d, max_len)) return 0;
    return part_bytes(b, heads, kv_heads, d, max_len);
}

int ecasq_attend(const void *q, int64_t q_row, int64_t q_head, int64_t b, int32_t heads, const ecasq_cache_t *k,
                 const ecasq_cache_t *v, const int32_t *table, int64_t table_row, const int32_t *lengths,
                 const int32_t *starts, int64_t max_len, float scale, void *out, int64_t out_row, int64_t out_head,
                 float *lse, void *ws, size_t ws_bytes, int32_t *status, ecasq_stream_t stream) {
    if (!cache_ok(k) || !cache_ok(v) || k->type != v->type || k->levels_n != v->levels_n || k->d != v->d ||
        k->heads != v->heads || k->pages != v->pages || k->page_size != v->page_size ||
        !sizes_ok(b, heads, k->heads, k->d, max_len))
        return ECASQ_EINVAL;
    if (b == 0) return ECASQ_OK;
    if (!q || !out || !lengths || (max_len && (!table || table_row < cdiv(max_len, k->page_size)))) return ECASQ_EINVAL;
    AttendArgs a{};
    a.q = q;
    a.out = out;
    a.table = table;
    a.lengths = lengths;
    a.starts = starts;
    a.lse = lse;
    a.status = status;
    const int64_t e = k->levels_n ? 1 : type_size(k->type);
    a.k = static_cast<const char *>(k->rows);
    a.v = static_cast<const char *>(v->rows);
    a.kt = static_cast<const char *>(k->levels);
    a.vt = static_cast<const char *>(v->levels);
    a.k_page = (uint64_t)(k->row_page * e);
    a.k_slot = (uint64_t)(k->row_slot * e);
    a.k_head = (uint64_t)(k->row_head * e);
    a.v_page = v->row_page * e;
    a.v_slot = v->row_slot * e;
    a.v_head = v->row_head * e;
    a.kt_page = k->level_page * 2;
    a.kt_slot = k->level_slot * 2;
    a.kt_head = k->level_head * 2;
    a.vt_page = v->level_page * 2;
    a.vt_slot = v->level_slot * 2;
    a.vt_head = v->level_head * 2;
    a.q_row = q_row;
    a.q_head = q_head;
    a.out_row = out_row;
    a.out_head = out_head;
    a.table_row = table_row;
    a.pages = k->pages;
    a.scale2 = scale * kLog2e;
    a.heads = heads;
    a.group = heads / k->heads;
    a.htiles = (int32_t)cdiv(a.group, kHeads);
    a.d = k->d;
    a.page_size = k->page_size;
    a.max_len = (int32_t)max_len;
    a.ws = ws;
    a.ws_bytes = ws_bytes;
    const FastDiv div(k->page_size);
    a.div_mul = div.mul;
    a.div_shift = div.shift;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool bf16 = k->type == ECASQ_BF16;
    int rc;
    if (k->type == ECASQ_F32) rc = launch_attend_f32(a, b, st);
    else if (!k->levels_n) rc = launch_attend_16(a, bf16, b, st);
    else if (k->levels_n == 8) rc = launch_attend_coded8(a, bf16, b, st);
    else rc = launch_attend_coded16(a, bf16, b, st);
    if (rc || a.splits == 1 || a.cluster) return rc;
    if (k->type == ECASQ_F32) return launch_join<float>(a, b, st);
    return bf16 ? launch_join<__nv_bfloat16>(a, b, st) : launch_join<__half>(a, b, st);
}

}  // extern "C"
