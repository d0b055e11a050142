// matvec_f32.cu -- ecasq_matvec for fp32.
//
// A block takes a run of rows and up to eight rows of x, which lie in shared memory.  Its 16 warps share the 128-column
// blocks of a tile of sixteen rows and, where there are few of those, take several tiles at once; a stage of the ring
// holds those tiles' rows, brought in by one bulk copy a row a few stages ahead, and one barrier a stage joins the sums
// and frees it.  The products are FMAs: a lane holds all eight columns for its share of k.
//
// What bounds it: no unit is full (issue slots 41 %, shared memory 30 %); sixteen warps an SM wait in turn for their lookups, the scales
// read from memory and the round's barrier.  The table of fp32 pairs is held once for each two lanes,
// so a lookup takes two transactions where the 16-bit types need one, and each eight weights read x once for every row of
// x.  8192 x 8192 by one row takes 29.1 us (1.2 TB/s), by eight 99 us; 2999 x 2050 by three 8.9 us.
#include <algorithm>

#include "matvec.cuh"

namespace ecasq {

constexpr int kMostStages = 4, kTableBytes = 256 * 128, kSumBytes = 2 * kWarps * 16 * 8 * 4, kBarBytes = 64, kLostAt = 8 * kMostStages;
constexpr int kRowPad = 64;  // a row's room in a stage is its bytes and this: two rows' reads do not meet in a bank

// Entry `byte J of w` of the table of pairs; l: the address of the lane's copy of entry 0.
template <int J> __device__ __forceinline__ float2 pair32(uint32_t w, uint32_t l) {
    return *static_cast<const float2 *>(__cvta_shared_to_generic((w >> 8 * J & 255u) * 128 + l));
}

// A warp's part of a row tile.
struct Sums {
    float p[2][8];  // all eight columns, of this lane's share of k; finish() leaves the layout above in c
    float c[4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; i++) p[0][i] = p[1][i] = 0.f;
    }
    __device__ __forceinline__ void add(const Sums &o, float sa, float sb) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            p[0][i] = fmaf(sa, o.p[0][i], p[0][i]);
            p[1][i] = fmaf(sb, o.p[1][i], p[1][i]);
        }
    }
    // Adds eight columns: codes wa of row g and wb of row g + 8, x from xs on.
    __device__ __forceinline__ void word(uint32_t wa, uint32_t wb, uint32_t l, const float *xs, int pitch, int nb) {
        const float2 va[4] = {pair32<0>(wa, l), pair32<1>(wa, l), pair32<2>(wa, l), pair32<3>(wa, l)};
        const float2 vb[4] = {pair32<0>(wb, l), pair32<1>(wb, l), pair32<2>(wb, l), pair32<3>(wb, l)};
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (i >= nb) break;
            const float4 x0 = *reinterpret_cast<const float4 *>(xs + i * pitch), x1 = *reinterpret_cast<const float4 *>(xs + i * pitch + 4);
            const float xv[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
            for (int j = 0; j < 4; j++) {
                p[0][i] = fmaf(va[j].y, xv[2 * j + 1], fmaf(va[j].x, xv[2 * j], p[0][i]));
                p[1][i] = fmaf(vb[j].y, xv[2 * j + 1], fmaf(vb[j].x, xv[2 * j], p[1][i]));
            }
        }
    }
    __device__ __forceinline__ void finish(int t) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float keep = t & 2 ? p[u][i + 4] : p[u][i], give = t & 2 ? p[u][i] : p[u][i + 4];
                w[i] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float keep = t & 1 ? w[i + 2] : w[i], give = t & 1 ? w[i] : w[i + 2];
                c[2 * u + i] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
            }
        }
    }
};

// WIDE: a scale group holds whole 128-column blocks (8192 x 8192 by one row, groups of 128: 29.9 us, and 33.0 without).
// Of a gated matrix a tile is eight rows of the gate and the same eight of the other half.
template <bool WIDE, After AFTER>
__global__ void __launch_bounds__(kThreads, 1) k_matvec_f32(const __grid_constant__ MatvecArgs a) {
    constexpr bool kTwo = AFTER == kGated;
    constexpr int kTile = kTwo ? 8 : 16;  // outputs of a tile
    extern __shared__ __align__(128) char smem[];
    char *table = smem;
    float *sums = reinterpret_cast<float *>(smem + kTableBytes);
    const uint32_t bars = smem_at(smem + kTableBytes + kSumBytes);
    char *rest = smem + kTableBytes + kSumBytes + kBarBytes;
    float *row_sums = reinterpret_cast<float *>(rest);  // [kRowsMost][8], only with several passes
    if (a.chunk < a.k) rest += kRowSumBytes;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t entry0 = smem_at(table) + 8 * (lane & 15);
    const int wk = wid & (a.warps_k - 1), wr = wid / a.warps_k, tiles = kWarps / a.warps_k, rows_at_once = 16 * tiles, outputs = kTile * tiles;
    const int i0 = 8 * blockIdx.y, nb = min(8, a.b - i0);
    float *xs = reinterpret_cast<float *>(rest);  // x, a.chunk columns a row
    const char *ring = rest + nb * a.chunk * 4;
    const int pitch = a.chunk / 2 + kRowPad, stage_bytes = rows_at_once * pitch;
    const int64_t r0 = row_of(a, blockIdx.x, gridDim.x);
    const int rows = (int)(row_of(a, blockIdx.x + 1, gridDim.x) - r0), rounds = (rows + outputs - 1) / outputs;
    const uint8_t *codes = a.codes + r0 * a.code_row;
    const float *scales = static_cast<const float *>(a.scales) + r0 * a.scale_row;

    wait_before();
    const uint32_t lost_at = bars + kLostAt;
    if (tid == 0) {
        for (int s = 0; s < a.stages; s++) bar_init(bars + 8 * s);
        set_word(lost_at, a.lost);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();

    uint32_t parity = 0;  // of the stages' next waits, a bit each
    bool lost = false;    // a wait of the block ran out
    int turn = 0;
    for (int64_t k0 = 0; k0 < a.k && !lost; k0 += a.chunk) {
        const int cols = (int)min((int64_t)a.chunk, a.k - k0), blocks = (cols + 127) / 128;
        if (k0) __syncthreads();
        auto fetch = [&](int round, int s) {
            const int first = round * outputs, count = min(outputs, rows - first), output = kTwo ? tid / 16 * 8 + (tid & 7) : tid;
            if (tid == 0) bar_expect(bars + 8 * s, count * (16 / kTile) * blocks * 64);
            if (tid < rows_at_once && output < count)
                bulk_copy(smem_at(ring + s * stage_bytes + tid * pitch), codes + (first + output + (kTwo ? (tid >> 3 & 1) * a.second : 0)) * a.code_row + k0 / 2, blocks * 64, bars + 8 * s);
        };
        for (int s = 0; s < a.stages && s < rounds; s++) fetch(s, s);

        // The codebook's pairs: warp w the sixteen with the second level w, half of the lanes a copy each.
        if (k0 == 0) {
            const float mine = (lane & 15) < a.m ? static_cast<const float *>(a.levels)[lane & 15] : 0.f;
            const float high = __shfl_sync(0xffffffffu, mine, wid);
#pragma unroll
            for (int j = 0; j < 16; j++) {
                const float low = __shfl_sync(0xffffffffu, mine, j);
                if (lane < 16) reinterpret_cast<float2 *>(table)[16 * (16 * wid + j) + lane] = make_float2(low, high);
            }
        }
        // Scales of rows g and g + 8, for the lane's words t of a block (WIDE: for the block), read one block ahead.  Rows beyond
        // the run repeat its last one; their sums are not stored.
        float next_a, next_b;
        auto next_scales = [&](int round, int at) {
            const int row = round * outputs + kTile * wr + g;
            const uint32_t w = group_of(a, (uint32_t)(k0 / 32) + 4 * at + (WIDE ? 0 : t));
            next_a = scales[min(row, rows - 1) * a.scale_row + w];
            next_b = scales[(kTwo ? min(row, rows - 1) + a.second : min(row + 8, rows - 1)) * a.scale_row + w];
        };
        next_scales(0, wk);
        // x, zero beyond k.
        const float *x = static_cast<const float *>(a.x) + i0 * a.x_row + k0;
        for (int i = 0; i < nb; i++)
            for (int c = tid; c < 128 * blocks; c += kThreads) xs[i * a.chunk + c] = c < cols ? x[i * a.x_row + c] : 0.f;
        __syncthreads();

        for (int round = 0, s = 0; round < rounds; round++) {
            if (!bar_wait(bars + 8 * s, parity >> s & 1)) set_word(lost_at, round + 1);
            parity ^= 1u << s;
            const char *tile = ring + s * stage_bytes + (16 * wr + g) * pitch + 16 * t;
            Sums acc;
            acc.clear();
            for (int at = wk; at < blocks; at += a.warps_k) {
                const float fa = next_a, fb = next_b;
                if (at + a.warps_k < blocks) next_scales(round, at + a.warps_k);
                else if (round + 1 < rounds) next_scales(round + 1, wk);
                const uint4 la = *reinterpret_cast<const uint4 *>(tile + 64 * at), lb = *reinterpret_cast<const uint4 *>(tile + 64 * at + 8 * pitch);
                const uint32_t wa[4] = {la.x, la.y, la.z, la.w}, wb[4] = {lb.x, lb.y, lb.z, lb.w};
                Sums part;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    if (i == 0 || !WIDE) part.clear();
                    part.word(wa[i], wb[i], entry0, xs + 128 * at + 32 * i + 8 * t, a.chunk, nb);
                    if (!WIDE) acc.add(part, __shfl_sync(0xffffffffu, fa, (lane & ~3) | i), __shfl_sync(0xffffffffu, fb, (lane & ~3) | i));
                }
                if (WIDE) acc.add(part, fa, fb);
            }
            acc.finish(t);
            float *buf = sums + turn * kWarps * 128;
            float *mine = buf + wid * 128 + 8 * g + 2 * t;
            *reinterpret_cast<float2 *>(mine) = make_float2(acc.c[0], acc.c[1]);
            *reinterpret_cast<float2 *>(mine + 64) = make_float2(acc.c[2], acc.c[3]);
            __syncthreads();
            lost = lost_by(lost_at, round);
            if (lost) {
                drain_ahead(bars, parity, s, round, rounds, a.stages);
                break;
            }
            if (round + a.stages < rounds) fetch(round + a.stages, s);
            // The tiles' sums over their warps: 16 rows of 8 columns each.
            for (int i = tid; i < 8 * outputs; i += kThreads) {
                float v = 0.f, u = 0.f;
                const int at = round * outputs + i / 8, col = i & 7;
                const bool there = at < rows && col < nb, last = there && k0 + a.chunk >= a.k;
                const float bias = last ? bias_of<float, AFTER>(a, r0 + at) : 0.f, residual = last ? residual_of<float, AFTER>(a, i0 + col, r0 + at) : 0.f;
                const float *from = buf + i / (8 * kTile) * a.warps_k * 128 + i % (8 * kTile);
                for (int w = 0; w < a.warps_k; w++) {
                    v += from[w * 128];
                    if (kTwo) u += from[w * 128 + 64];
                }
                if (there) {
                    if (a.chunk < a.k) {
                        if (k0) v += row_sums[at * 8 + col];
                        row_sums[at * 8 + col] = v;
                        if (kTwo) {
                            if (k0) u += row_sums[kRowsMost / 2 * 8 + at * 8 + col];
                            row_sums[kRowsMost / 2 * 8 + at * 8 + col] = u;
                        }
                    }
                    if (last) static_cast<float *>(a.y)[(i0 + col) * a.y_row + r0 + at] = result<float, AFTER>(a, v, u, bias, residual);
                }
            }
            turn ^= 1;  // the next round's sums go to the other half: one barrier a round
            s = s + 1 == a.stages ? 0 : s + 1;
        }
    }
    if (lost) {  // all of the block's results are NaN
        drain_lost(bars, parity, a.stages);
        __syncthreads();  // behind what it has stored
        if (tid == 0 && a.status) atomicOr(a.status, ECASQ_BAD_WAIT);
        for (int i = tid; i < 8 * rows; i += kThreads)
            if ((i & 7) < nb) static_cast<float *>(a.y)[(i0 + (i & 7)) * a.y_row + r0 + i / 8] = CUDART_NAN_F;
    }
}

template <After AFTER> static int launch_f32(MatvecArgs &a, int32_t group, cudaStream_t st) {
    const int64_t blocks = row_blocks(a.n, AFTER == kGated ? kRowsMost / 2 : kRowsMost), tiles = cdiv(cdiv(cdiv(a.n, 8), blocks), AFTER == kGated ? 1 : 2), kb = cdiv(a.k, 128), nb = std::min(a.b, 8);
    const int64_t room = 227 * 1024 - kTableBytes - kSumBytes - kBarBytes - kRowSumBytes;
    // The warps' split between columns and row tiles that leaves the fullest warp the least; of equal ones that with the
    // fewest warps a tile, whose sums have to be joined.
    int64_t best = INT64_MAX;
    for (int w = kWarps; w >= 1; w /= 2) {
        const int64_t cost = cdiv(kb, w) * cdiv(tiles, kWarps / w);
        if (w < kWarps && (w > kb ? cost >= best : cost > best)) continue;
        best = cost;
        a.warps_k = w;
    }
    // Two stages at least, and x.
    const int64_t at_once = 16 * (kWarps / a.warps_k);
    auto stage = [&](int64_t chunk) { return at_once * (64 * chunk + kRowPad); };
    int64_t chunk = kb;
    while (chunk > 1 && nb * chunk * 512 + 2 * stage(chunk) > room) chunk--;
    a.chunk = (int32_t)(128 * chunk);
    const int64_t x_bytes = nb * chunk * 512;
    a.stages = (int32_t)std::min<int64_t>(std::min<int64_t>(kMostStages, (room - x_bytes) / stage(chunk)), cdiv(tiles, kWarps / a.warps_k));
    const int smem = (int)(227 * 1024 - room - (a.chunk < a.k ? 0 : kRowSumBytes) + x_bytes + a.stages * stage(chunk));
    static std::atomic<int> allowed[2][kDevices];
    const bool wide = group % 128 == 0;
    auto *kernel = wide ? k_matvec_f32<true, AFTER> : k_matvec_f32<false, AFTER>;
    const int rc = allow_smem(kernel, 227 * 1024, allowed[wide]);
    if (rc) return rc;
    return launch_early(kernel, dim3((unsigned)blocks, (unsigned)cdiv(a.b, 8)), kThreads, smem, st, a);
}

int launch_matvec_f32(MatvecArgs &a, After after, int32_t group, cudaStream_t st) {
    if (after == kGated) return launch_f32<kGated>(a, group, st);
    return after == kProject ? launch_f32<kProject>(a, group, st) : launch_f32<kPlain>(a, group, st);
}

}  // namespace ecasq
