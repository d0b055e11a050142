// matvec.cu -- products with a matrix of 4-bit codes (ecasq_pack, ecasq_matvec).
#include <algorithm>
#include <cstring>
#include <type_traits>

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
    int32_t *status;
    int64_t x_row, code_row, scale_row, y_row, n, k;
    int32_t b, m, groups;
    int32_t warps_k;              // warps that share a row tile along k, a power of two; the others take other tiles
    int32_t chunk;                // columns that one pass over the rows covers, a multiple of 128
    int32_t stages;               // stages of the codes' ring
    uint32_t div_mul, div_shift;  // words of 32 columns to scale groups: w div (group / 32), as umulhi(w, div_mul) >> div_shift
                                  // or w >> div_shift if div_mul is 0
};

// One block takes a run of rows and up to eight rows of x.  Its 16 warps share the 128-column blocks of a tile of
// sixteen rows and, where there are few of those, take several tiles at once; a stage of the ring holds those tiles' rows,
// brought in by one bulk copy a row a few stages ahead, and one barrier a stage joins the sums and frees it.
//
// What bounds it: the codes' bytes in the end, and on the way there shared memory and the issue slots: a byte of codes is
// two weights, and one lookup in a table of all 256 pairs of levels gives both.  The table is held once a lane
// (entry e of lane l at word 32 e + l), so that no two lanes meet in a bank; 32 lookups, 8 transactions for the
// codes themselves and up to 8 for the scales stand, for each KB of codes, against the 44 clocks that memory needs for it.
//
// 16-bit types: a pair of weights is an operand register of mma.m16n8k16 as it stands, with the rows of x as its
// eight columns and fp32 sums.  The order of the columns within a product is free, and the packed layout is
// made for it: a lane (g, t) = (lane / 4, lane mod 4) reads 16 bytes of row g, words t, t + 4, t + 8 and t + 12 of the
// block, so that one step of all lanes covers 32 neighbouring columns, which lie in one scale group; the scale is
// applied to the fp32 sums of its group.  A warp keeps to its R blocks for all rows, with their x in registers.
// (With one to eight columns there is no reuse that a larger tensor tile could draw on.)
// fp32: the same lookups in a table of fp32 pairs, held once for each two lanes, x in shared memory, and FMAs.
constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kRowsMost = 512;  // rows of a block
constexpr int kMostStages = 4;
constexpr int kTableBytes = 256 * 128, kSumBytes = 2 * kWarps * 16 * 8 * 4, kRowSumBytes = kRowsMost * 8 * 4, kBarBytes = 64;
constexpr int kRowPad = 64;     // a row's room in a stage is its bytes and this: two rows' reads do not meet in a bank
constexpr int kSpins = 1 << 18; // of a wait, each of a microsecond or so

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool wait_full(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < kSpins; i++) {
        uint32_t done;
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done) : "r"(bar), "r"(parity), "r"(1000) : "memory");
        if (done) return true;
    }
    return false;
}
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
// Entry `byte j of w` of the table of pairs; l: the address of the lane's copy of entry 0.  The address is left to the integer
// multiply-add, as the permutes already fill their own pipe.
template <int J> __device__ __forceinline__ uint32_t entry_at(uint32_t w, uint32_t l) {
    uint32_t byte, at;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(byte) : "r"(w), "n"(0x4440 | J));
    asm("mad.lo.u32 %0, %1, 128, %2;" : "=r"(at) : "r"(byte), "r"(l));
    return at;
}
template <int J> __device__ __forceinline__ uint32_t pair16(uint32_t w, uint32_t l) {
    uint32_t v;
    asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(entry_at<J>(w, l)));
    return v;
}
template <int J> __device__ __forceinline__ float2 pair32(uint32_t w, uint32_t l) {
    float2 v;
    asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(entry_at<J>(w, l)));
    return v;
}

// A warp's part of a row tile: 16 rows, and of the eight columns the two of its lane.
// c[0], c[1]: row g, columns 2t, 2t + 1; c[2], c[3]: row g + 8.
template <typename T> struct Sums {
    float c[4];
    __device__ __forceinline__ void clear() { c[0] = c[1] = c[2] = c[3] = 0.f; }
    __device__ __forceinline__ void add(const Sums &o, float sa, float sb) {
        c[0] = fmaf(sa, o.c[0], c[0]);
        c[1] = fmaf(sa, o.c[1], c[1]);
        c[2] = fmaf(sb, o.c[2], c[2]);
        c[3] = fmaf(sb, o.c[3], c[3]);
    }
    // Eight more columns (FIRST: the first): codes wa of row g and wb of row g + 8, xv those of row g of x.
    template <bool FIRST> __device__ __forceinline__ void word(uint32_t wa, uint32_t wb, uint32_t l, const uint32_t (&xv)[4]) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        if (FIRST) mma_pairs<T>(c, zero, pair16<0>(wa, l), pair16<0>(wb, l), pair16<1>(wa, l), pair16<1>(wb, l), xv[0], xv[1]);
        else mma_pairs<T>(c, c, pair16<0>(wa, l), pair16<0>(wb, l), pair16<1>(wa, l), pair16<1>(wb, l), xv[0], xv[1]);
        mma_pairs<T>(c, c, pair16<2>(wa, l), pair16<2>(wb, l), pair16<3>(wa, l), pair16<3>(wb, l), xv[2], xv[3]);
    }
    __device__ __forceinline__ void finish(int) {}
};
template <> struct Sums<float> {
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
    template <bool FIRST> __device__ __forceinline__ void word(uint32_t wa, uint32_t wb, uint32_t l, const float *xs, int pitch, int nb) {
        if (FIRST) clear();
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

// WIDE: a scale group holds whole 128-column blocks.  R: blocks of a warp in a chunk at most (16-bit types).
template <typename T, typename S, bool WIDE, int R>
__global__ void __launch_bounds__(kThreads, 1) k_matvec(const __grid_constant__ MatvecArgs a) {
    extern __shared__ __align__(128) char smem[];
    constexpr bool kF32 = sizeof(T) == 4;
    char *table = smem;
    const uint32_t entry0 = smem_at(table) + (kF32 ? 8 * (threadIdx.x & 15) : 4 * (threadIdx.x & 31));
    float *sums = reinterpret_cast<float *>(smem + kTableBytes);
    const uint32_t bars = smem_at(smem + kTableBytes + kSumBytes);
    char *rest = smem + kTableBytes + kSumBytes + kBarBytes;
    float *row_sums = reinterpret_cast<float *>(rest);  // [kRowsMost][8], only with several chunks
    if (a.chunk < a.k) rest += kRowSumBytes;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const int wk = wid & (a.warps_k - 1), wr = wid / a.warps_k, tiles = kWarps / a.warps_k, rows_at_once = 16 * tiles;
    const int i0 = 8 * blockIdx.y, nb = min(8, a.b - i0);
    T *xs = reinterpret_cast<T *>(rest);  // fp32: x, a.chunk columns a row
    if (kF32) rest += nb * a.chunk * 4;
    const char *ring = rest;
    const int pitch = a.chunk / 2 + kRowPad, stage_bytes = rows_at_once * pitch;
    // Runs of whole eights of rows, as even as they can be.
    const int64_t units = (a.n + 7) / 8;
    const int64_t r0 = units * blockIdx.x / gridDim.x * 8;
    const int rows = (int)(min(a.n, units * (blockIdx.x + 1) / gridDim.x * 8) - r0), rounds = (rows + rows_at_once - 1) / rows_at_once;
    const uint8_t *codes = a.codes + r0 * a.code_row;
    const S *scales = static_cast<const S *>(a.scales) + r0 * a.scale_row;

    if (tid == 0)
        for (int s = 0; s < a.stages; s++) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * s) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();

    uint32_t parity = 0;  // of the stages' next waits, a bit each
    bool lost = false;    // a wait ran out
    int turn = 0;
    for (int64_t k0 = 0; k0 < a.k; k0 += a.chunk) {
        const int cols = (int)min((int64_t)a.chunk, a.k - k0), blocks = (cols + 127) / 128;
        const int own = wk < blocks ? (blocks - wk + a.warps_k - 1) / a.warps_k : 0;  // this warp's blocks
        if (k0) __syncthreads();
        auto fetch = [&](int round, int s) {
            const int first = round * rows_at_once, count = min(rows_at_once, rows - first);
            if (tid == 0)
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bars + 8 * s), "r"(count * blocks * 64) : "memory");
            if (tid < count)
                asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                 smem_at(ring + s * stage_bytes + tid * pitch)),
                             "l"(codes + (first + tid) * a.code_row + k0 / 2), "r"(blocks * 64), "r"(bars + 8 * s)
                             : "memory");
        };
        for (int s = 0; s < a.stages && s < rounds; s++) fetch(s, s);

        // Scales of a round's tile, fetched a round ahead: of rows g and g + 8, for the lane's words t of each block (WIDE: for
        // the block).  Rows beyond the run repeat its last one; their sums are not stored.
        constexpr int kHeld = kF32 ? 1 : R;
        S sa[kHeld], sb[kHeld];
        auto scale_at = [&](int r) {
            uint32_t w = (uint32_t)(k0 / 32) + 4 * (wk + r * a.warps_k) + (WIDE ? 0 : t);
            w = a.div_mul ? __umulhi(w, a.div_mul) >> a.div_shift : w >> a.div_shift;
            return min(w, (uint32_t)a.groups - 1);
        };
        uint32_t at[kHeld];
#pragma unroll
        for (int r = 0; r < kHeld; r++) at[r] = scale_at(r);
        auto rows_of = [&](int round, const S *&qa, const S *&qb) {
            const int row = round * rows_at_once + 16 * wr + g;
            qa = scales + min(row, rows - 1) * a.scale_row;
            qb = scales + min(row + 8, rows - 1) * a.scale_row;
        };
        auto fetch_scales = [&](int round) {
            const S *qa, *qb;
            rows_of(round, qa, qb);
#pragma unroll
            for (int r = 0; r < kHeld; r++) {
                sa[r] = qa[at[r]];
                sb[r] = qb[at[r]];
            }
        };
        if (!kF32) fetch_scales(0);

        // The codebook's pairs: warp w the sixteen with the second level w, a lane a copy.
        if (k0 == 0) {
            const T mine = (lane & 15) < a.m ? static_cast<const T *>(a.levels)[lane & 15] : from_f32<T>(0.f);
            uint32_t bits = 0;
            memcpy(&bits, &mine, sizeof(T));
            const uint32_t high = __shfl_sync(0xffffffffu, bits, wid);
#pragma unroll
            for (int j = 0; j < 16; j++) {
                const uint32_t low = __shfl_sync(0xffffffffu, bits, j);
                const int e = 16 * wid + j;
                if constexpr (kF32) {
                    if (lane < 16) reinterpret_cast<uint2 *>(table)[16 * e + lane] = make_uint2(low, high);
                } else {
                    reinterpret_cast<uint32_t *>(table)[32 * e + lane] = low | high << 16;
                }
            }
        }
        // x, zero beyond k.
        const T *x = static_cast<const T *>(a.x) + i0 * a.x_row + k0;
        uint32_t xr[kHeld][4][4];
        if constexpr (kF32) {
            for (int i = 0; i < nb; i++)
                for (int c = tid; c < 128 * blocks; c += kThreads) xs[i * a.chunk + c] = c < cols ? x[i * a.x_row + c] : from_f32<T>(0.f);
        } else {
            const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (nb == 1 || a.x_row % 8 == 0);
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int c = 128 * (wk + r * a.warps_k) + 32 * i + 8 * t;
                    const T *from = x + g * a.x_row + c;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (g < nb && c < cols) {
                        if (vec && c + 8 <= cols) {
                            v = *reinterpret_cast<const uint4 *>(from);
                        } else {
                            alignas(16) T one[8];
#pragma unroll
                            for (int j = 0; j < 8; j++) one[j] = c + j < cols ? from[j] : from_f32<T>(0.f);
                            v = *reinterpret_cast<const uint4 *>(one);
                        }
                    }
                    xr[r][i][0] = v.x;
                    xr[r][i][1] = v.y;
                    xr[r][i][2] = v.z;
                    xr[r][i][3] = v.w;
                }
        }
        __syncthreads();

        for (int round = 0, s = 0; round < rounds; round++) {
            if (!wait_full(bars + 8 * s, parity >> s & 1)) lost = true;
            parity ^= 1u << s;
            const char *tile = ring + s * stage_bytes + (16 * wr + g) * pitch + 64 * wk + 16 * t;
            Sums<T> acc;
            acc.clear();
            // One block: its codes, its scales, and word(first, i, codes a, codes b), which adds columns 32 i ...
            auto block = [&](const char *p, float fa, float fb, auto &&word) {
                const uint4 la = *reinterpret_cast<const uint4 *>(p), lb = *reinterpret_cast<const uint4 *>(p + 8 * pitch);
                const uint32_t wa[4] = {la.x, la.y, la.z, la.w}, wb[4] = {lb.x, lb.y, lb.z, lb.w};
                Sums<T> part;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    if (i == 0 || !WIDE) word(part, std::true_type(), i, wa[i], wb[i]);
                    else word(part, std::false_type(), i, wa[i], wb[i]);
                    if (!WIDE) acc.add(part, __shfl_sync(0xffffffffu, fa, (lane & ~3) | i), __shfl_sync(0xffffffffu, fb, (lane & ~3) | i));
                }
                if (WIDE) acc.add(part, fa, fb);
            };
            if constexpr (kF32) {
                const S *qa, *qb;
                rows_of(round, qa, qb);
                for (int r = 0; r < own; r++) {
                    const uint32_t w = scale_at(r);
                    const T *xb = xs + 128 * (wk + r * a.warps_k) + 8 * t;
                    block(tile + 64 * r * a.warps_k, to_f32(qa[w]), to_f32(qb[w]), [&](Sums<T> &part, auto first, int i, uint32_t wa, uint32_t wb) {
                        part.template word<decltype(first)::value>(wa, wb, entry0, xb + 32 * i, a.chunk, nb);
                    });
                }
            } else {
                float fa[R], fb[R];
#pragma unroll
                for (int r = 0; r < R; r++) {
                    fa[r] = to_f32(sa[r]);
                    fb[r] = to_f32(sb[r]);
                }
                if (round + 1 < rounds) fetch_scales(round + 1);
                // (All R blocks, without a branch between them: x is zero where there is none.)
#pragma unroll
                for (int r = 0; r < R; r++)
                        block(tile + 64 * r * a.warps_k, fa[r], fb[r], [&](Sums<T> &part, auto first, int i, uint32_t wa, uint32_t wb) {
                            part.template word<decltype(first)::value>(wa, wb, entry0, xr[r][i]);
                        });
            }
            acc.finish(t);
            float *buf = sums + turn * kWarps * 128;
            float *mine = buf + wid * 128 + 8 * g + 2 * t;
            *reinterpret_cast<float2 *>(mine) = make_float2(acc.c[0], acc.c[1]);
            *reinterpret_cast<float2 *>(mine + 64) = make_float2(acc.c[2], acc.c[3]);
            __syncthreads();
            if (round + a.stages < rounds) fetch(round + a.stages, s);
            // The tiles' sums over their warps: 16 rows of 8 columns each.
            for (int i = tid; i < 128 * tiles; i += kThreads) {
                float v = 0.f;
                const float *from = buf + (i >> 7) * a.warps_k * 128 + (i & 127);
                for (int w = 0; w < a.warps_k; w++) v += from[w * 128];
                const int row = round * rows_at_once + i / 8, col = i & 7;
                if (row < rows && col < nb) {
                    if (a.chunk < a.k) {
                        if (k0) v += row_sums[row * 8 + col];
                        row_sums[row * 8 + col] = v;
                    }
                    if (k0 + a.chunk >= a.k) static_cast<T *>(a.y)[(i0 + col) * a.y_row + r0 + row] = from_f32<T>(lost ? CUDART_NAN_F : v);
                }
            }
            turn ^= 1;  // the next round's sums go to the other half: one barrier a round
            s = s + 1 == a.stages ? 0 : s + 1;
        }
    }
    if (lost && a.status) atomicOr(a.status, ECASQ_BAD_WAIT);
}

template <typename T, typename S, int R>
static int launch_matvec_blocks(const MatvecArgs &a, bool wide, int smem, int64_t blocks, cudaStream_t st) {
    auto *kernel = wide ? k_matvec<T, S, true, R> : k_matvec<T, S, false, R>;
    ECASQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    note_launch();
    kernel<<<dim3((unsigned)blocks, (unsigned)cdiv(a.b, 8)), kThreads, smem, st>>>(a);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
}

template <typename T, typename S>
static int launch_matvec(MatvecArgs &a, int32_t group, cudaStream_t st) {
    constexpr bool f32 = sizeof(T) == 4;
    // One block for each SM (152), more where a block would have over kRowsMost rows.
    const int64_t units = cdiv(a.n, 8), blocks = std::max(std::min<int64_t>(units, 152), cdiv(units, kRowsMost / 8));
    const int64_t tiles = cdiv(cdiv(units, blocks), 2), kb = cdiv(a.k, 128);
    const int64_t room = 227 * 1024 - kTableBytes - kSumBytes - kBarBytes - kRowSumBytes, nb = std::min(a.b, 8);
    // The warps' split between columns and row tiles that leaves the fullest warp the least; of equal ones that with the
    // fewest warps a tile, whose sums have to be joined.  A warp holds x for four blocks at most (fp32: any number).
    int64_t best = INT64_MAX;
    for (int w = kWarps; w >= 1; w /= 2) {
        const int64_t cost = cdiv(kb, w) * cdiv(tiles, kWarps / w);
        if (w < kWarps && (w > kb ? cost >= best : cost > best || (!f32 && cdiv(kb, w) > 4))) continue;
        best = cost;
        a.warps_k = w;
    }
    const int64_t at_once = 16 * (kWarps / a.warps_k), own = f32 ? 1 : std::min<int64_t>(cdiv(kb, a.warps_k), 4);  // blocks of a warp in a chunk
    // A stage and, in fp32, x: bytes a column.  Two stages at least.
    auto stage = [&](int64_t chunk) { return at_once * (chunk / 2 + kRowPad); };
    if (f32) {
        int64_t chunk = kb;
        while (chunk > 1 && nb * chunk * 512 + 2 * stage(128 * chunk) > room) chunk--;
        a.chunk = (int32_t)(128 * chunk);
    } else {
        a.chunk = (int32_t)(128 * own * a.warps_k);
    }
    const int64_t x_bytes = f32 ? nb * a.chunk * 4 : 0;
    a.stages = (int32_t)std::min<int64_t>(std::min<int64_t>(kMostStages, (room - x_bytes) / stage(a.chunk)), cdiv(tiles, kWarps / a.warps_k));
    const int smem = (int)(227 * 1024 - room - (a.chunk < a.k ? 0 : kRowSumBytes) + x_bytes + a.stages * stage(a.chunk));
    const bool wide = group % 128 == 0;
    if (own == 1) return launch_matvec_blocks<T, S, 1>(a, wide, smem, blocks, st);
    if constexpr (!f32) {
        if (own == 2) return launch_matvec_blocks<T, S, 2>(a, wide, smem, blocks, st);
        if (own == 3) return launch_matvec_blocks<T, S, 3>(a, wide, smem, blocks, st);
        return launch_matvec_blocks<T, S, 4>(a, wide, smem, blocks, st);
    }
    return ECASQ_EINVAL;
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
                 int64_t k, int32_t group, void *y, int64_t y_row, int32_t *status, ecasq_stream_t stream) {
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
    const FastDiv div(group / 32);
    a.div_mul = div.mul;
    a.div_shift = div.shift;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool scales32 = scale_type == ECASQ_F32;
    if (type == ECASQ_F32) return launch_matvec<float, float>(a, group, st);
    if (type == ECASQ_F16) return scales32 ? launch_matvec<__half, float>(a, group, st) : launch_matvec<__half, __half>(a, group, st);
    return scales32 ? launch_matvec<__nv_bfloat16, float>(a, group, st) : launch_matvec<__nv_bfloat16, __nv_bfloat16>(a, group, st);
}

}  // extern "C"
