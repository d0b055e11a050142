// matvec.cu -- products with a matrix of 4-bit codes (ecasq_pack, ecasq_matvec): the packing, the kernel for 16-bit types.
#include <algorithm>

#include "matvec.cuh"

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

// 16-bit types.  A block takes a run of rows and up to eight rows of x.  A warp keeps to R neighbouring 128-column blocks,
// whose x it holds in registers, and runs down the rows, a tile of sixteen at a time; with few columns the warps take
// several tiles at once.  A stage of the ring holds a round's rows, brought in by one bulk copy a row a round or more ahead;
// a barrier a round joins the warps' sums and frees its stage.  The rows' scales come a round ahead too, by cp.async in the
// 16-byte pieces that hold them (loads to registers are waited for together with the lookups: 39.6 against 36.8 us for 28672 x
// 8192 by eight rows).  More columns than the warps cover take several passes, or two or four blocks of a cluster take a slice of
// the columns each and add their sums over the cluster, which also fills the card where rows are few (393 x 15530 by two rows: 7.2 us
// by clusters, 14.7 in passes of single blocks; 8192 x 28672 by eight: 41.5 and 51.2).
//
// A pair of weights is an operand register of mma.m16n8k16 as it stands, with the rows of x as its eight columns and
// fp32 sums; the order of the columns within a product is free.  (With one to eight columns there is no reuse that a
// larger tensor tile could draw on; more rows of x take a pass over the matrix for each eight, where there would be.)
//
// What bounds it: the codes' bytes in the end, and on the way there the latency of lookups and products at sixteen warps an
// SM (issue slots 45 %, shared memory 46 %, DRAM 35 % busy with eight rows).  28672 x 8192 by eight rows of bf16 takes 35.5 us,
// 3.5 TB/s; 8192 x 8192 by one row of fp16, groups of 64, 15.2 us, 2.4 TB/s; a small matrix 3.5 us: the launch, one memory latency
// and the table.  The table is held once a lane, so that no two lanes meet in a bank; 32 lookups, 8 transactions for the codes
// themselves and up to 8 for the scales stand, for each KB of codes, against the 44 clocks that memory needs for it.  Entry e of lane l lies at address
// kTableAt + 256 e + 4 l: one byte permute puts the code byte between the lane's constant ones, and that is the address.
constexpr int kTableAt = 0x20000, kAboveAt = 0x30000, kSmemBytes = 227 * 1024;
constexpr int kBarBytes = 64, kMostStages = 4, kLostAt = 8 * kMostStages;  // barriers, and the word of lost waits
constexpr int kWindowMost = 2048;  // where a block's own shared memory begins at most (it is 1 KB)
constexpr int kBelowRoom = kTableAt - kWindowMost - kBarBytes, kAboveRoom = kSmemBytes - kAboveAt;

// d = c + A B
template <typename T> __device__ __forceinline__ void mma_pairs(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma_pairs<__half>(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
template <> __device__ __forceinline__ void mma_pairs<__nv_bfloat16>(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// Entry `byte J of w` of the table of pairs; l: the address of the lane's copy of entry 0, whose byte 1 is zero.
template <int J> __device__ __forceinline__ uint32_t pair16(uint32_t w, uint32_t l) {
    uint32_t at;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(at) : "r"(w), "r"(l), "n"(0x7604 | J << 4));
    return *static_cast<const uint32_t *>(__cvta_shared_to_generic(at));
}

// Of eight 16-bit values the first `count`, zeros for the others.
__device__ __forceinline__ void keep(uint4 &v, int count) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; j++) w[j] = count >= 2 * j + 2 ? w[j] : count == 2 * j + 1 ? w[j] & 0xffffu : 0;
    v = make_uint4(w[0], w[1], w[2], w[3]);
}
// The eight that begin `skip` bytes into the pieces lo and hi.
__device__ __forceinline__ uint4 eight_of(const uint4 &lo, const uint4 &hi, int skip) {
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int j = 0; j < 6; j++) w[j] = skip & 8 ? w[j + 2] : w[j];
#pragma unroll
    for (int j = 0; j < 5; j++) w[j] = skip & 4 ? w[j + 1] : w[j];
#pragma unroll
    for (int j = 0; j < 4; j++) w[j] = skip & 2 ? __funnelshift_r(w[j], w[j + 1], 16) : w[j];
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// WIDE: a scale group holds whole 128-column blocks, so that a block's products are one sum (8192 x 8192 by eight rows, groups of
// 128: 15.9 us, and 16.9 with a sum for each 32 columns).
template <typename T, typename S, bool WIDE, int R>
__global__ void __launch_bounds__(kThreads, 1) k_matvec(const __grid_constant__ MatvecArgs a) {
    extern __shared__ __align__(128) char smem[];
    const uint32_t base = smem_at(smem), bars = base, window = base & 0xff000000u;  // (a cluster's blocks have windows 2^24 apart)
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    float *row_sums = reinterpret_cast<float *>(smem + kBarBytes);  // [kRowsMost][8], with several passes or slices
    char *scale_ring = smem + kBarBytes + (a.keep ? kRowSumBytes : 0), *table = smem + (kTableAt + window - base), *above = smem + (kAboveAt + window - base);
    const uint32_t entry0 = window + kTableAt + 4 * lane;
    const int wk = wid & (a.warps_k - 1), wr = wid / a.warps_k, tiles_at_once = kWarps / a.warps_k;
    const int i0 = 8 * blockIdx.y, nb = min(8, a.b - i0);
    const unsigned run = blockIdx.x / a.slices, runs = gridDim.x / a.slices, rank = blockIdx.x % a.slices;
    const int64_t r0 = row_of(a, run, runs);
    const uint32_t k_first = rank * a.slice, k_end = min((uint32_t)a.k, k_first + a.slice);
    const int rows = (int)(row_of(a, run + 1, runs) - r0), tiles = (rows + 15) / 16, rounds = (tiles + tiles_at_once - 1) / tiles_at_once;
    const S *scales = static_cast<const S *>(a.scales) + r0 * a.scale_row;
    // A stage is two pieces, the rows 0 .. 7 and 8 .. 15 of its tiles; as many pieces as fit lie below the table, the others above.
    char *below = scale_ring + 32 * tiles_at_once * a.scale_pitch;  // two rounds' scales
    const int piece_bytes = 8 * tiles_at_once * a.pitch, pieces_below = a.pieces_below;
    auto piece_at = [&](int p) -> char * { return p < pieces_below ? below + p * piece_bytes : above + (p - pieces_below) * piece_bytes; };
    // The sums of a round, 128 for each warp, lie in the halves of the table's rows that it does not use: 32 floats each, two
    // rounds in turn.
    auto sum_at = [&](int i) -> float * { return reinterpret_cast<float *>(table + (i >> 5) * 256 + 128 + (i & 31) * 4); };

    wait_before();
    // (Loads are issued before anything waits for another's: the levels here, x before the table is built.)
    const T level = (lane & 15) < a.m ? static_cast<const T *>(a.levels)[lane & 15] : from_f32<T>(0.f);
    const uint32_t lost_at = bars + kLostAt;
    if (tid == 0) {
        for (int s = 0; s < a.stages; s++) bar_init(bars + 8 * s);
        set_word(lost_at, a.lost);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();

    uint32_t parity = 0;  // of the stages' next waits, a bit each
    int turn = 0;
    for (uint32_t k0 = k_first; k0 < k_end; k0 += a.chunk) {
        const int cols = min(a.chunk, (int)(k_end - k0)), blocks = (cols + 127) / 128;
        // A warp brings in one row of each tile.
        const int fetch_row = 16 * lane + wid;
        auto fetch = [&](int round, int s) {
            const int first = round * 16 * tiles_at_once, count = min(16 * tiles_at_once, rows - first);
            if (tid == 0) bar_expect(bars + 8 * s, count * blocks * 64);
            if (lane < tiles_at_once && fetch_row < count)
                bulk_copy(smem_at(piece_at(2 * s + (wid >> 3))) + (8 * lane + (wid & 7)) * a.pitch, a.codes + (r0 + first + fetch_row) * a.code_row + k0 / 2, blocks * 64,
                          bars + 8 * s);
        };
        for (int s = 0; s < a.stages && s < rounds; s++) fetch(s, s);

        // A round's scales: of each row the pieces that hold its groups first .. last.  A warp takes a row of each tile.
        const uint32_t first_group = group_of(a, k0 / 32), last_group = group_of(a, (k0 + cols - 1) / 32);
        const int scale_bytes = (int)(last_group - first_group + 1) * (int)sizeof(S);
        auto fetch_scales = [&](int round) {
            const int first = round * 16 * tiles_at_once;
            for (int row = wid; row < 16 * tiles_at_once && first + row < rows; row += kWarps) {
                const uintptr_t from = reinterpret_cast<uintptr_t>(scales + (first + row) * a.scale_row + first_group);
                const uint32_t to = smem_at(scale_ring) + ((round & 1) * 16 * tiles_at_once + row) * a.scale_pitch;
                for (int at = 16 * lane; at < (int)(from & 15) + scale_bytes; at += 512)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + at), "l"((from & ~(uintptr_t)15) + at));
            }
        };
        fetch_scales(0);
        // Where the lane's scales lie among a row's: of its words t of each block (WIDE: of the block).
        int at[R];
#pragma unroll
        for (int r = 0; r < R; r++) at[r] = (int)(min(group_of(a, k0 / 32 + 4 * (wk * R + r) + (WIDE ? 0 : t)), last_group) - first_group) * (int)sizeof(S);

        // x, zero beyond k.
        uint4 xr[R][4];
        {
            const T *x = static_cast<const T *>(a.x) + (i0 + min(g, nb - 1)) * a.x_row + k0;
            const int have = g < nb ? cols - 128 * wk * R - 8 * t : 0;  // values from the lane's first on
            const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.b == 1 || a.x_row % 8 == 0);
            if (vec) {
#pragma unroll
                for (int r = 0; r < R; r++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        xr[r][i] = 128 * r + 32 * i < have ? *reinterpret_cast<const uint4 *>(x + 128 * (wk * R + r) + 32 * i + 8 * t) : make_uint4(0, 0, 0, 0);
                if (cols % 8)
#pragma unroll
                    for (int r = 0; r < R; r++)
#pragma unroll
                        for (int i = 0; i < 4; i++) keep(xr[r][i], have - 128 * r - 32 * i);
            } else {
                // In the 16-byte pieces that hold them, two blocks' at a time, and without a branch between the loads (value by
                // value each load would wait for the one before: 16.0 against 13.3 us for 2046 x 8508 by five rows).
                const int skip = (int)(reinterpret_cast<uintptr_t>(x) & 15);
                const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(x) & ~(uintptr_t)15);
#pragma unroll
                for (int r0 = 0; r0 < R; r0 += 2) {
                    uint4 lo[2][4], hi[2][4];
#pragma unroll
                    for (int r = 0; r < 2 && r0 + r < R; r++)
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const int count = have - 128 * (r0 + r) - 32 * i, at = count > 0 ? 16 * (wk * R + r0 + r) + 4 * i + t : 0;
                            lo[r][i] = p[at];
                            hi[r][i] = p[count > 0 && skip + 2 * count > 16 ? at + 1 : at];
                        }
#pragma unroll
                    for (int r = 0; r < 2 && r0 + r < R; r++)
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            xr[r0 + r][i] = eight_of(lo[r][i], hi[r][i], skip);
                            keep(xr[r0 + r][i], have - 128 * (r0 + r) - 32 * i);
                        }
                }
            }
        }
        // The codebook's pairs: warp w the sixteen with the second level w, a lane a copy.
        if (k0 == k_first) {
            const uint32_t bits = reinterpret_cast<const uint16_t &>(level), high = __shfl_sync(0xffffffffu, bits, wid);
#pragma unroll
            for (int j = 0; j < 16; j++)
                reinterpret_cast<uint32_t *>(table + 256 * (16 * wid + j))[lane] = __shfl_sync(0xffffffffu, bits, j) | high << 16;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();

#pragma unroll 1
        for (int round = 0, s = 0; round < rounds; round++) {
            if (round + 1 < rounds) fetch_scales(round + 1);
            // The scales of rows g and g + 8 (rows beyond the run have none; their sums are not stored).
            const int row = 16 * wr + g;
            const char *mine = scale_ring + ((round & 1) * 16 * tiles_at_once + row) * a.scale_pitch;
            const uint32_t row0 = (uint32_t)reinterpret_cast<uintptr_t>(scales + first_group), step = (uint32_t)a.scale_row * sizeof(S);
            const char *qa = mine + (row0 + (round * 16 * tiles_at_once + row) * step & 15), *qb = mine + 8 * a.scale_pitch + (row0 + (round * 16 * tiles_at_once + row + 8) * step & 15);
            if (!bar_wait(bars + 8 * s, parity >> s & 1)) set_word(lost_at, round + 1);
            parity ^= 1u << s;
            const char *up = piece_at(2 * s) + (8 * wr + g) * a.pitch + 64 * R * wk + 16 * t, *low = piece_at(2 * s + 1) + (8 * wr + g) * a.pitch + 64 * R * wk + 16 * t;
            float c[4] = {0.f, 0.f, 0.f, 0.f};  // c[0], c[1]: row g, columns 2t, 2t + 1; c[2], c[3]: row g + 8
            // (All R blocks, without a branch between them: x is zero where there is none.  A warp without any rests.)
            if (wk * R < blocks)
#pragma unroll
            for (int r = 0; r < R; r++) {
                const uint4 la = *reinterpret_cast<const uint4 *>(up + 64 * r), lb = *reinterpret_cast<const uint4 *>(low + 64 * r);
                const uint32_t wa[4] = {la.x, la.y, la.z, la.w}, wb[4] = {lb.x, lb.y, lb.z, lb.w};
                const float zero[4] = {0.f, 0.f, 0.f, 0.f}, fa = to_f32(*reinterpret_cast<const S *>(qa + at[r])), fb = to_f32(*reinterpret_cast<const S *>(qb + at[r]));
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t a0 = pair16<0>(wa[i], entry0), a1 = pair16<0>(wb[i], entry0), a2 = pair16<1>(wa[i], entry0), a3 = pair16<1>(wb[i], entry0);
                    if (i == 0 || !WIDE) mma_pairs<T>(p, zero, a0, a1, a2, a3, xr[r][i].x, xr[r][i].y);
                    else mma_pairs<T>(p, p, a0, a1, a2, a3, xr[r][i].x, xr[r][i].y);
                    mma_pairs<T>(p, p, pair16<2>(wa[i], entry0), pair16<2>(wb[i], entry0), pair16<3>(wa[i], entry0), pair16<3>(wb[i], entry0), xr[r][i].z, xr[r][i].w);
                    if (i == 3 || !WIDE) {
                        const float ra = WIDE ? fa : __shfl_sync(0xffffffffu, fa, (lane & ~3) | i);
                        const float rb = WIDE ? fb : __shfl_sync(0xffffffffu, fb, (lane & ~3) | i);
                        c[0] = fmaf(ra, p[0], c[0]);
                        c[1] = fmaf(ra, p[1], c[1]);
                        c[2] = fmaf(rb, p[2], c[2]);
                        c[3] = fmaf(rb, p[3], c[3]);
                    }
                }
            }
            if (2 * t < nb) {
                float *own = sum_at((turn * kWarps + wid) * 128 + 8 * g + 2 * t);
                *reinterpret_cast<float2 *>(own) = make_float2(c[0], c[1]);
                *reinterpret_cast<float2 *>(own + 128) = make_float2(c[2], c[3]);  // 64 sums on: two rows of the table
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncthreads();
            if (round + a.stages < rounds) {
                if (lost_by(lost_at, round)) {
                    drain_ahead(bars, parity, s, round, rounds, a.stages);
                    break;
                }
                fetch(round + a.stages, s);
            }
            // The tiles' sums over their warps, 16 rows of 8 columns each; four warps a tile, others each round.
            for (int i = (tid + 128 * round) & (kThreads - 1); i < 128 * tiles_at_once; i += kThreads) {
                const int row = round * 16 * tiles_at_once + i / 8, col = i & 7;
                if (row < rows && col < nb) {
                    const float *of = sum_at((turn * kWarps + (i >> 7) * a.warps_k) * 128 + (i & 127));
                    float v = 0.f;
#pragma unroll 8
                    for (int w = 0; w < a.warps_k; w++) v += of[w * 256];  // 128 sums on: four rows of the table
                    if (a.keep) {
                        if (k0 > k_first) v += row_sums[row * 8 + col];
                        row_sums[row * 8 + col] = v;
                    }
                    if (a.slices == 1 && k0 + a.chunk >= k_end) static_cast<T *>(a.y)[(i0 + col) * a.y_row + r0 + row] = from_f32<T>(v);
                }
            }
            turn ^= 1;  // the next round's sums go to the other half
            s = s + 1 == a.stages ? 0 : s + 1;
        }
        if (k0 + a.chunk < k_end && __syncthreads_or(get_word(lost_at))) break;  // (a barrier: the sums of this pass, before the next one's)
    }
    if (get_word(lost_at)) {  // all of the block's results are NaN
        drain_lost(bars, parity, a.stages);
        __syncthreads();  // behind what it has stored
        if (tid == 0 && a.status) atomicOr(a.status, ECASQ_BAD_WAIT);
        for (int i = tid; i < 8 * rows; i += kThreads) {
            if (a.slices > 1) row_sums[i] = CUDART_NAN_F;
            else if ((i & 7) < nb) static_cast<T *>(a.y)[(i0 + (i & 7)) * a.y_row + r0 + i / 8] = from_f32<T>(CUDART_NAN_F);
        }
    }
    if (a.slices > 1) {  // each block adds its share of the rows over the cluster
        cluster_barrier();
        for (int i = (int)rank * kThreads + tid; i < 8 * rows; i += a.slices * kThreads) {
            const int row = i / 8, col = i & 7;
            if (col >= nb) continue;
            float v = 0.f;
            for (int s = 0; s < a.slices; s++) {
                float of;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(of) : "r"(of_rank(smem_at(row_sums + i), s)) : "memory");
                v += of;
            }
            static_cast<T *>(a.y)[(i0 + col) * a.y_row + r0 + row] = from_f32<T>(v);
        }
        cluster_barrier();
    }
}

// Whether a block's own shared memory begins where kBelowRoom takes it to: asked once a device.
static int window_ok() {
    static std::atomic<int> known[kDevices];
    int device = 0, reserved = 0;
    ECASQ_CUDA_TRY(cudaGetDevice(&device));
    if (device < kDevices && known[device].load(std::memory_order_acquire)) return ECASQ_OK;
    ECASQ_CUDA_TRY(cudaDeviceGetAttribute(&reserved, cudaDevAttrReservedSharedMemoryPerBlock, device));
    if (reserved > kWindowMost) return ECASQ_ECUDA;
    if (device < kDevices) known[device].store(1, std::memory_order_release);
    return ECASQ_OK;
}

template <typename T, typename S, bool WIDE, int R>
static int launch_matvec_blocks(const MatvecArgs &a, int64_t runs, cudaStream_t st) {
    static std::atomic<int> allowed[kDevices];
    int rc = window_ok();
    if (!rc) rc = allow_smem(k_matvec<T, S, WIDE, R>, kSmemBytes, allowed);
    if (rc) return rc;
    return launch_clusters(k_matvec<T, S, WIDE, R>, dim3((unsigned)(runs * a.slices), (unsigned)cdiv(a.b, 8)), dim3((unsigned)a.slices), kThreads, kSmemBytes, st, a);
}

// Clusters of c = 2 or 4 blocks that the card holds at once (76 and 36), asked once a device.  Every k_matvec has the same threads and
// shared memory.
static int clusters_held(int c, int *held) {
    static std::atomic<int> known[2][kDevices], allowed[kDevices];
    int device = 0;
    ECASQ_CUDA_TRY(cudaGetDevice(&device));
    *held = device < kDevices ? known[c / 4][device].load(std::memory_order_acquire) : 0;
    if (*held > 0) return ECASQ_OK;
    auto *kernel = k_matvec<__half, __half, false, 1>;
    const int rc = allow_smem(kernel, kSmemBytes, allowed);
    if (rc) return rc;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ECASQ_CUDA_TRY(cudaOccupancyMaxActiveClusters(held, kernel, &cfg));
    if (*held < 1) return ECASQ_ECUDA;
    if (device < kDevices) known[c / 4][device].store(*held, std::memory_order_release);
    return ECASQ_OK;
}

template <typename T, typename S>
static int launch_matvec(MatvecArgs &a, int32_t group, cudaStream_t st) {
    // (32-bit arithmetic: this runs in every call.)
    const auto over = [](int v, int by) { return (v + by - 1) / by; };
    const int eights = (int)cdiv(a.n, 8), all = (int)cdiv(a.k, 128);
    // The split of the columns over a cluster, of the warps between columns and row tiles, and the blocks a warp, that take the
    // least time: passes over the rows, each with about three blocks' time until its first codes are there, rounds, and the
    // blocks of a round, which costs about half a block of its own; more where the next round's codes have no stage to come
    // into; and the cluster's barriers.
    int64_t best = INT64_MAX, runs = 0;
    int own = 0;
    for (int c = 1; c <= 4; c *= 2) {
        const int kb = over(all, c);
        int at_once_most = 152;
        if (c > 1) {
            if (best <= 12 || a.b > 8 || (c - 1) * kb >= all) break;  // (12: the least cost of a cluster)
            const int rc = clusters_held(c, &at_once_most);
            if (rc) return rc;
        }
        const int blocks = std::max(std::min(eights, at_once_most), over(eights, kRowsMost / 8)), tiles = over(over(eights, blocks), 2);
        for (int w = kWarps; w >= 1; w /= 2) {
            const int rounds = over(tiles, kWarps / w), at_once = 16 * (kWarps / w);
            for (int r = 4; r >= 1; r--) {
                const int passes = over(kb, w * r), chunk = 128 * r * w;
                const bool keep = passes > 1 || c > 1;
                int64_t cost = (int64_t)over(blocks, at_once_most) * passes * (rounds * (2 * r + 1) + 6) + (c > 1 ? 3 : 0);
                if (cost >= best) continue;
                // A row's room in a stage: its bytes, and what makes it an odd multiple of 64, so that two rows' reads do not meet in
                // a bank; its scales' room: the pieces of 16 bytes that may hold them, and an odd multiple of 16.
                const int pitch = chunk / 2 + (r * w % 2 ? 0 : 64), piece = at_once / 2 * pitch;
                const int groups = std::min(a.groups, chunk / group + 2), scale_pitch = (groups * (int)sizeof(S) + 30) / 32 * 32 + 16;
                const int left = kBelowRoom - (keep ? kRowSumBytes : 0) - 2 * at_once * scale_pitch;
                if (left < 0) continue;
                const int below = left / piece, stages = std::min({(below + kAboveRoom / piece) / 2, rounds, kMostStages});
                if (stages < 2 && rounds > 1) cost *= 2;
                if (stages < 1 || cost >= best) continue;
                best = cost;
                own = r;
                runs = blocks;
                a.slices = c;
                a.slice = c > 1 ? 128 * kb : (int32_t)a.k;
                a.keep = keep;
                a.warps_k = w;
                a.chunk = chunk;
                a.pitch = pitch;
                a.scale_pitch = scale_pitch;
                a.stages = stages;
                a.pieces_below = below;
            }
        }
    }
    if (best == INT64_MAX) return ECASQ_EINVAL;  // (no size leads here: one block a warp always fits)
    switch (2 * own + (group % 128 == 0)) {
        case 2: return launch_matvec_blocks<T, S, false, 1>(a, runs, st);
        case 3: return launch_matvec_blocks<T, S, true, 1>(a, runs, st);
        case 4: return launch_matvec_blocks<T, S, false, 2>(a, runs, st);
        case 5: return launch_matvec_blocks<T, S, true, 2>(a, runs, st);
        case 6: return launch_matvec_blocks<T, S, false, 3>(a, runs, st);
        case 7: return launch_matvec_blocks<T, S, true, 3>(a, runs, st);
        case 8: return launch_matvec_blocks<T, S, false, 4>(a, runs, st);
        default: return launch_matvec_blocks<T, S, true, 4>(a, runs, st);
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
    const bool scales32 = scale_type == ECASQ_F32;
    if (type == ECASQ_F32) return launch_matvec_f32(a, group, st);
    if (type == ECASQ_F16) return scales32 ? launch_matvec<__half, float>(a, group, st) : launch_matvec<__half, __half>(a, group, st);
    return scales32 ? launch_matvec<__nv_bfloat16, float>(a, group, st) : launch_matvec<__nv_bfloat16, __nv_bfloat16>(a, group, st);
}

}  // extern "C"
