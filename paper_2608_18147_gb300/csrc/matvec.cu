// matvec.cu -- products with a matrix of 4-bit codes (ecasq_pack, ecasq_matvec).
#include <algorithm>

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
    int64_t x_row, code_row, scale_row, y_row, n, k;
    int32_t b, m, groups;
    int32_t warps_k;              // warps that share a row tile along k, a power of two
    int32_t chunk;                // columns of x in shared memory at a time, a multiple of 128
    int32_t x_pitch;              // elements from one row of x to the next there
    uint32_t div_mul, div_shift;  // words of 32 columns to scale groups: w div (group / 32), as umulhi(w, div_mul) >> div_shift
                                  // or w >> div_shift if div_mul is 0
};

// One block takes a run of rows, sixteen at a time, and up to eight rows of x; its warps share a tile's 128-column
// blocks and, where there are few of those, its tiles.
//
// What bounds it: the codes' bytes in the end, and on the way there shared memory: a byte of codes is two weights, and
// one lookup in a table of all 256 pairs of levels gives both.  The table is held once a lane (entry e of
// lane l at word 32 e + l), so that no two lanes meet in a bank; 32 lookups, 4 to 16 reads of x and the
// codes' own 8 transactions for each KB of codes stand against the 44 clocks that memory needs for it.
//
// 16-bit types: a pair of weights is an operand register of mma.m16n8k16 as it stands, with the rows of x as its
// eight columns and fp32 sums.  The order of the columns within a product is free, and the packed layout is
// made for it: a lane (g, t) = (lane / 4, lane mod 4) loads 16 bytes of row g, words t, t + 4, t + 8 and t + 12 of the
// block, so that one step of all lanes covers 32 neighbouring columns, which lie in one scale group; the scale is
// applied to the fp32 sums of its group.  (With one to eight columns there is no reuse that a larger tensor
// tile could draw on.)
// fp32: the same lookups in a table of fp32 pairs, held once for each two lanes, and FMAs.
constexpr int kWarps = 16, kThreads = 32 * kWarps, kDepth = 4;  // kDepth: 1 KB loads that a warp has in flight
constexpr int kRowsMost = 512;                                 // rows of a block
constexpr int kTableBytes = 256 * 128, kSumBytes = 2 * kWarps * 16 * 8 * 4, kRowSumBytes = kRowsMost * 8 * 4;

__device__ __forceinline__ uint4 load_codes(const uint8_t *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename T> __device__ __forceinline__ void mma_pairs(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma_pairs<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma_pairs<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
    // Adds eight columns: codes wa of row g and wb of row g + 8, x at xs (row g of x; only read if g < nb).
    __device__ __forceinline__ void word(uint32_t wa, uint32_t wb, const char *table, const T *xs, int, int lane, int nb) {
        uint4 xv = make_uint4(0, 0, 0, 0);
        if ((lane >> 2) < nb) xv = *reinterpret_cast<const uint4 *>(xs);
        const uint32_t l4 = 4 * lane;
        auto look = [&](uint32_t byte7) { return *reinterpret_cast<const uint32_t *>(table + ((byte7 & 0x7f80u) | l4)); };
        mma_pairs<T>(c, look(wa << 7), look(wb << 7), look(wa >> 1), look(wb >> 1), xv.x, xv.y);
        mma_pairs<T>(c, look(wa >> 9), look(wb >> 9), look(wa >> 17), look(wb >> 17), xv.z, xv.w);
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
    __device__ __forceinline__ void word(uint32_t wa, uint32_t wb, const char *table, const float *xs, int pitch, int lane, int nb) {
        const uint32_t l8 = 8 * (lane & 15);
        float2 va[4], vb[4];
        auto look = [&](uint32_t byte7) { return *reinterpret_cast<const float2 *>(table + ((byte7 & 0x7f80u) | l8)); };
        va[0] = look(wa << 7);
        va[1] = look(wa >> 1);
        va[2] = look(wa >> 9);
        va[3] = look(wa >> 17);
        vb[0] = look(wb << 7);
        vb[1] = look(wb >> 1);
        vb[2] = look(wb >> 9);
        vb[3] = look(wb >> 17);
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

// WIDE: a scale group holds whole 128-column blocks.
template <typename T, typename S, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) k_matvec(const __grid_constant__ MatvecArgs a) {
    extern __shared__ __align__(128) char smem[];
    constexpr bool kF32 = sizeof(T) == 4;
    char *table = smem;
    float *sums = reinterpret_cast<float *>(smem + kTableBytes);
    float *row_sums = sums + kSumBytes / 4;  // [kRowsMost][8], only with several chunks
    T *xs = reinterpret_cast<T *>(smem + kTableBytes + kSumBytes + (a.chunk < a.k ? kRowSumBytes : 0));
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    const int wk = wid & (a.warps_k - 1), wr = wid / a.warps_k, tiles_apart = kWarps / a.warps_k;
    const int i0 = 8 * blockIdx.y, nb = min(8, a.b - i0);
    // Runs of whole eights of rows, as even as they can be.
    const int64_t units = (a.n + 7) / 8;
    const int64_t r0 = units * blockIdx.x / gridDim.x * 8, r1 = min(a.n, units * (blockIdx.x + 1) / gridDim.x * 8);
    const int tiles = (int)((r1 - r0 + 15) / 16);
    const S *scales = static_cast<const S *>(a.scales);

    struct Load {
        uint4 a, b;
        float sa, sb;
    } ring[kDepth];
    for (int64_t k0 = 0; k0 < a.k; k0 += a.chunk) {
        const int cols = (int)min((int64_t)a.chunk, a.k - k0), blocks = (cols + 127) / 128;
        const bool some = wk < blocks;  // a last chunk may have fewer blocks than warps_k
        // Two walks over (tile, block), one ahead for the loads.
        int ahead_tile = wr, ahead_block = wk;
        auto load = [&](Load &l) {
            if (ahead_tile < tiles) {
                const int64_t ra = r0 + 16 * ahead_tile + g, rb = ra + 8;
                const int64_t at = (k0 + 128 * ahead_block) / 2 + 16 * t;
                uint32_t w = (uint32_t)(k0 / 32) + 4 * ahead_block + (WIDE ? 0 : t);
                w = a.div_mul ? __umulhi(w, a.div_mul) >> a.div_shift : w >> a.div_shift;
                w = min(w, (uint32_t)a.groups - 1);
                l.a = l.b = make_uint4(0, 0, 0, 0);
                l.sa = l.sb = 0.f;
                if (some && ra < r1) {
                    l.a = load_codes(a.codes + ra * a.code_row + at);
                    l.sa = to_f32(scales[ra * a.scale_row + w]);
                }
                if (some && rb < r1) {
                    l.b = load_codes(a.codes + rb * a.code_row + at);
                    l.sb = to_f32(scales[rb * a.scale_row + w]);
                }
                ahead_block += a.warps_k;
                if (ahead_block >= blocks) {
                    ahead_block = wk;
                    ahead_tile += tiles_apart;
                }
            }
        };
#pragma unroll
        for (int s = 0; s < kDepth; s++) load(ring[s]);

        // The codebook's pairs and the chunk of x, zero beyond k.
        if (k0 == 0) {
            const T *levels = static_cast<const T *>(a.levels);
            constexpr int kCopies = kF32 ? 16 : 32;
            for (int i = tid; i < 256 * kCopies; i += kThreads) {
                const int e = i / kCopies, lo = e & 15, hi = e >> 4;
                const T zero = from_f32<T>(0.f);
                reinterpret_cast<T *>(table)[2 * i] = lo < a.m ? levels[lo] : zero;
                reinterpret_cast<T *>(table)[2 * i + 1] = hi < a.m ? levels[hi] : zero;
            }
        } else {
            __syncthreads();
        }
        const T *x = static_cast<const T *>(a.x) + i0 * a.x_row + k0;
        constexpr int kVec = 16 / sizeof(T);
        const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (nb == 1 || a.x_row % kVec == 0);
        for (int i = 0; i < nb; i++)
            for (int c = kVec * tid; c < 128 * blocks; c += kVec * kThreads) {
                alignas(16) T v[kVec];
                T *to = xs + i * a.x_pitch + c;
                if (vec && c + kVec <= cols) {
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(x + i * a.x_row + c));
                    continue;
                }
#pragma unroll
                for (int j = 0; j < kVec; j++) v[j] = c + j < cols ? x[i * a.x_row + c + j] : from_f32<T>(0.f);
                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(v);
            }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();

        int tile = wr, block = wk, turn = 0;
        Sums<T> acc;
        acc.clear();
        const T *mine = xs + (kF32 ? 0 : g * a.x_pitch) + 8 * t;
        while (tile < tiles) {
#pragma unroll
            for (int s = 0; s < kDepth; s++) {
                if (tile < tiles) {
                    const Load &l = ring[s];
                    const uint32_t wa[4] = {l.a.x, l.a.y, l.a.z, l.a.w}, wb[4] = {l.b.x, l.b.y, l.b.z, l.b.w};
                    const T *xb = mine + 128 * block;
                    Sums<T> part;
                    if (some) {
                        if (WIDE) part.clear();
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            if (!WIDE) part.clear();
                            part.word(wa[i], wb[i], table, xb + 32 * i, a.x_pitch, lane, nb);
                            if (!WIDE) acc.add(part, __shfl_sync(0xffffffffu, l.sa, (lane & ~3) | i), __shfl_sync(0xffffffffu, l.sb, (lane & ~3) | i));
                        }
                        if (WIDE) acc.add(part, l.sa, l.sb);
                    }
                    load(ring[s]);
                    block += a.warps_k;
                    if (block >= blocks) {  // the tile's sums over its warps
                        acc.finish(t);
                        float *buf = sums + (turn * kWarps + wr * a.warps_k) * 128;
                        float *own = buf + wk * 128 + 8 * g + 2 * t;
                        *reinterpret_cast<float2 *>(own) = make_float2(acc.c[0], acc.c[1]);
                        *reinterpret_cast<float2 *>(own + 64) = make_float2(acc.c[2], acc.c[3]);
                        if (a.warps_k > 1) asm volatile("bar.sync %0, %1;" ::"r"(wr + 1), "r"(32 * a.warps_k) : "memory");
                        else __syncwarp();
                        for (int i = 32 * wk + lane; i < 128; i += 32 * a.warps_k) {
                            float v = 0.f;
                            for (int w = 0; w < a.warps_k; w++) v += buf[w * 128 + i];
                            const int64_t row = r0 + 16 * tile + i / 8;
                            const int col = i & 7;
                            if (row < r1 && col < nb) {
                                if (a.chunk < a.k) {
                                    float *keep = row_sums + (16 * tile + i / 8) * 8 + col;
                                    if (k0) v += *keep;
                                    *keep = v;
                                }
                                if (k0 + a.chunk >= a.k) static_cast<T *>(a.y)[(i0 + col) * a.y_row + row] = from_f32<T>(v);
                            }
                        }
                        turn ^= 1;  // the next tile's sums go to the other half: one barrier a tile
                        block = wk;
                        tile += tiles_apart;
                        acc.clear();
                    }
                }
            }
        }
    }
}

// Shared memory for x: what is left beside the table and the sums.
constexpr int64_t kXBytes = 227 * 1024 - kTableBytes - kSumBytes;

template <typename T, typename S>
static int launch_matvec(MatvecArgs &a, int32_t group, cudaStream_t st) {
    const int nb = std::min(a.b, 8);
    // Rows of x lie 64 bytes off a multiple of 128 from one another, so that the reads of two rows do not meet in a bank.
    const int64_t pad = 64 / (int64_t)sizeof(T), wide = cdiv(a.k, 128) * 128;
    if (nb * (wide + pad) * (int64_t)sizeof(T) <= kXBytes) a.chunk = (int32_t)std::max(wide, a.k);
    else a.chunk = (int32_t)(((kXBytes - kRowSumBytes) / (nb * (int64_t)sizeof(T)) - pad) / 128 * 128);
    a.x_pitch = (int32_t)(std::min<int64_t>(a.chunk, wide) + pad);
    const int smem = kTableBytes + kSumBytes + (a.chunk < a.k ? kRowSumBytes : 0) + nb * a.x_pitch * (int)sizeof(T);
    // One block for each SM (152), more where a block would have over kRowsMost rows.
    const int64_t units = cdiv(a.n, 8), blocks = std::max(std::min<int64_t>(units, 152), cdiv(units, kRowsMost / 8));
    // The warps' split between columns and row tiles that leaves the fullest warp the least.
    const int64_t kb = std::min<int64_t>(a.chunk, wide) / 128, tiles = cdiv(cdiv(units, blocks), 2);
    int64_t best = INT64_MAX;
    for (int w = 1; w <= kWarps && w <= kb; w *= 2) {
        const int64_t cost = cdiv(kb, w) * cdiv(tiles, kWarps / w);
        if (cost <= best) {
            best = cost;
            a.warps_k = w;
        }
    }
    auto *kernel = group % 128 == 0 ? k_matvec<T, S, true> : k_matvec<T, S, false>;
    ECASQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    note_launch();
    kernel<<<dim3((unsigned)blocks, (unsigned)cdiv(a.b, 8)), kThreads, smem, st>>>(a);
    ECASQ_LAUNCH_CHECK();
    return ECASQ_OK;
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
                 int64_t k, int32_t group, void *y, int64_t y_row, ecasq_stream_t stream) {
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
