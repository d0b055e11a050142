// project_tc.cuh -- ecasq_project and ecasq_gated for more rows of x than a pass of the matrix-vector kernels takes.
//
// The matrix is the left operand: its codes become levels, which go to tensor memory as they are (16 bits, exact), 128 rows a
// block and 256 a pair of blocks; the rows of x are the right operand, in shared memory.  The sums of the columns of one scale group, 256 of them at most,
// come out of tensor memory, are multiplied by their row's scale, which is one number a thread there, and are added up in registers.  So
// products and scales are exact to fp32, as in ecasq_matvec.  (Levels times scales, rounded to 16 bits before the
// product, would need no sums in between, but are off by as much as the output's own rounding.)
//
// What bounds it (8192 x 8192 of bf16, groups of 128, by 4096 rows: 385 to 395 us, 1.4 PFLOP/s, three quarters of a library's 16-bit product on the same
// card): the tensor core is busy 59 % of the time.  At its rate a block of 128 columns of a pair's 256 x 256 tile is 1024 clocks; an adding warp took 740 for
// its share of a block's sums (eight loads of 16 columns from tensor memory, 92 clocks each, before two of them were under way at once), so smaller groups,
// with more sums, cost more: 551 us in groups of 64, 930 in groups of 32, 370 in groups of 256, and 380 in longer
// ones, whose sums are taken out as often.  With the results left unwritten it took 368 us: about 3 us for each of a pair's seven tiles.  A residual adds about 8 us a tile (447 us).  Registers
// spill in 21 of the 48 kernels, 12 bytes stored and 40 read in this case's.  With few rows of x it is the ways between the warps: where each block has a tile of its own, 128 columns take 0.38 us by 32 rows and 0.60 by 128 rows, on top of 6 us for the shortest product.  9700 x 8192 by 64 rows takes 25 us
// in single blocks and took 42 in pairs; where a pair has as many tiles as a block there is little to gain (8192 x 8192 by 16 rows 21 us both ways, by 128 rows 28 and 29).
#pragma once

#include <algorithm>
#include <type_traits>

#include "project.cuh"
#include "tc.cuh"

namespace ecasq {

struct TcArgs {
    const void *levels, *scales;
    void *y;
    int32_t *status;
    int64_t scale_row, y_row, n, b, k, second;  // second: the first row of a gated matrix's other half
    int32_t m, group, type, scale_type;
    int32_t blocks;         // blocks of 128 columns
    int32_t span_blocks;    // blocks whose sums are taken out together, where a scale group holds whole ones: spans begin at multiples of it, and groups too
    int32_t split;          // blocks of a cluster that share the columns; 1 for pairs
    int32_t x_tiles, w_tiles, tiles;  // tiles of rows of x; of the matrix's rows; of the product
    int32_t panel;          // tiles of rows of x that the tiles of the matrix's rows go by before the next ones
    bool wide;              // y and the residual in pieces of four values
    uint32_t none;          // 0, which the compiler does not know
    uint32_t lost;          // test hook: 1 where blocks begin as if a wait had run out
    Epilogue epi;
};

constexpr int kACols = 32;  // columns of tensor memory that 64 columns' levels take
constexpr int kCodeStage = 128 * 64, kSplitMost = 6;
constexpr int kScales = 8, kScaleLag = 6;  // scale groups in shared memory; of them on their way

// The tensor core's fp32 sums are cut off, not rounded, at each step of 16 columns, which makes them smaller by up to a unit in the last place a step.  So no sum stays there for more than
// kSpanMost blocks: in a group of 16384 columns of values of one sign sums were 5.3e-5 too small when they stayed for the whole group; they are 1.2e-6 too small taken out after two blocks, 0.55e-6 after one.
constexpr int kSpanMost = 2;

// fp32 operands are three bf16 terms, most significant first (8 bits each); of their nine products the six that reach 2^-16.  Each term's sums are taken out after every block.
__device__ __constant__ const int8_t kXTerm[6] = {0, 0, 0, 1, 1, 2}, kLevelTerm[6] = {0, 1, 2, 0, 1, 0};

// ND columns (rows of x) a product, NH of them a tile.  F32: fp32 operands as bf16 terms, whose levels are found by byte permutes; those of 16-bit
// types by lookups in a table of pairs.
template <int ND, int NH, bool GATED, bool F32> struct TcShape {
    static constexpr int kN = ND * NH;
    static constexpr int kDecodeWarps = NH == 2 ? 4 : 8, kWarps = 4 + kDecodeWarps + 8, kThreads = 32 * kWarps;
    // Two blocks of a cluster take 256 rows of the matrix together, and each brings half of the rows of x, where these are many; where they are few, and what
    // takes time are the ways between the warps, not the bytes, a block works alone: none of its barriers is another's.
    static constexpr bool kPair = kN > 128;
    static constexpr int kBlocks = kPair ? 2 : 1, kXRows = ND / kBlocks;  // rows of x that a block brings for one product
    static constexpr int kRows = (GATED ? 64 : 128) * kBlocks;            // outputs of a row of x in a tile
    static constexpr int kXStage = NH * kXRows * 256;
    static constexpr int kDBufs = ND == 128 ? 3 : ND == 64 ? 4 : 8;       // buffers for sums in tensor memory
    static constexpr int kAStages = ND == 128 ? 4 : 8, kAAt = 512 - kAStages * kACols;  // stages of levels, behind the sums
    static_assert(kAAt >= kDBufs * ND, "the sums' buffers end where the levels begin");
    static constexpr int kTable = F32 ? 0 : 256 * 128;            // a pair of levels for each byte of codes, a copy a lane
    static constexpr int kXStages = kN >= 256 ? 4 : kN == 128 ? 3 : kN == 64 ? 5 : 8, kCodeStages = kN >= 128 ? 3 : kN == 64 ? 9 : 12;
    // A wait for a barrier's phase ends at once where the phase before it has not ended either, so a warp may wait for a phase only if it knows of the one before.  The warps that decode are teams, which take
    // turns at the blocks: where they would also take turns at a stage of codes, each has barriers of its own for it, whose phases it has all waited for.  (With one barrier a stage a team went on with
    // the codes of three blocks before, and freed the stage for others, when the copy for the other team came later than both copies after it.)  Of a stage of x a team has waited for
    // its levels' stage before, which was free once the products of the block kAStages / 2 before, and all before them, had been done.  Of the three buffers of sums of a pair the two parts of a tile's rows of x
    // take turns too: sums are ready in the order of their products, so a part that has added up those two before knows of those three before.  (Barriers of their own for the parts took
    // 405 us where 8192 x 8192 by 4096 rows takes 385.)
    static constexpr int kTeams = kDecodeWarps / 4, kCodeBars = kCodeStages % kTeams ? kCodeStages * kTeams : kCodeStages;
    static_assert(kXStages % kTeams == 0 || kXStages >= kAStages / 2, "a team might wait for a phase of a stage of x and not know of the one before");
    static_assert(kAStages / 2 % kTeams == 0, "stages of levels are a team's own");
    static constexpr int kOwn = NH == 2 ? ND : ND / 2;            // columns of an adding thread
    static constexpr int kOut = NH == 2 ? 32 : kOwn;  // of them at a time on their way out through shared memory
    static constexpr int kSums = 2 * kOut * 128 * 4;              // what the adding warps have on their way out
    // Registers of a thread of the first four warps, of those that decode and of those that add; together no more than the block was launched with.
    static constexpr bool kUneven = kOwn >= 64;
    static constexpr int kRegs = 48, kDecodeRegs = 80, kAddRegs = NH == 2 ? 192 : 136;
    static_assert(4 * kRegs + kDecodeWarps * kDecodeRegs + 8 * kAddRegs <= kWarps * (65536 / kThreads / 8 * 8), "the split would wait for ever");
    static constexpr int kBars = 2 * kXStages + kCodeBars + kCodeStages + 2 * kAStages + 2 * kDBufs + 2 * kScales + 3;
    static constexpr int kTableAt = kXStages * kXStage + kCodeStages * kCodeStage, kSumsAt = kTableAt + kTable, kScalesAt = kSumsAt + kSums, kBooksAt = kScalesAt + kScales * 128 * 4, kBarsAt = kBooksAt + 128;
    static constexpr int kBytes = 1024 + kBarsAt + 8 * kBars + 16;  // 1024: to begin at a multiple of it
};

__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t s) {
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(s));
    return d;
}
// The levels of a word of eight codes, as four pairs.  t: the low bytes of levels 0-3, 4-7, 8-11, 12-15, then their high bytes.
// The lower and the upper eight levels are looked up by the codes' low three bits, and a permute that spreads the sign bits of w << 4 and w,
// which are the codes' fourth bits, chooses.
__device__ __forceinline__ void decode(uint32_t w, const uint32_t (&t)[8], uint32_t *to) {
    const uint32_t low3 = w & 0x77777777u, up = w << 4;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t s = h ? low3 >> 16 : low3, m = permute(up, w, h ? 0xFBEA : 0xD9C8);
        const uint32_t l0 = permute(t[0], t[1], s), l1 = permute(t[2], t[3], s), h0 = permute(t[4], t[5], s), h1 = permute(t[6], t[7], s);
        const uint32_t l = (l0 & ~m) | (l1 & m), hi = (h0 & ~m) | (h1 & m);
        to[2 * h] = permute(l, hi, 0x5140);
        to[2 * h + 1] = permute(l, hi, 0x7362);
    }
}

// Four neighbouring values of one of the 16-bit types, or of fp32, to fp32 and from it.
template <bool F32> using FourOf = std::conditional_t<F32, uint4, uint2>;
__device__ __forceinline__ void widen(const uint4 &p, bool, float (&v)[4]) {
    v[0] = __uint_as_float(p.x), v[1] = __uint_as_float(p.y), v[2] = __uint_as_float(p.z), v[3] = __uint_as_float(p.w);
}
__device__ __forceinline__ void widen(const uint2 &p, bool bf16, float (&v)[4]) {
    const uint32_t w[2] = {p.x, p.y};
#pragma unroll
    for (int i = 0; i < 2; i++) {
        if (bf16) {
            v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(reinterpret_cast<const __half2 &>(w[i]));
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
    }
}
__device__ __forceinline__ void narrow(const float (&v)[4], bool, uint4 &p) {
    p = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ void narrow(const float (&v)[4], bool bf16, uint2 &p) {
    if (bf16) {
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.x) : "f"(v[1]), "f"(v[0]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.y) : "f"(v[3]), "f"(v[2]));
    } else {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.x) : "f"(v[1]), "f"(v[0]));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.y) : "f"(v[3]), "f"(v[2]));
    }
}

// How four warps' sums leave the block.  They lie in shared memory, entry (column c, matrix row r of the block) at 128 c + r, and
// a thread takes four neighbouring outputs of a row of x, so that a row's 64 or 128 outputs leave side by side (each matrix row's outputs on their own, 64
// bytes a warp, took 60 us a tile of 256 x 256; eight a thread spill, as a thread's sums of the other columns are held meanwhile).  Of a gated
// matrix a warp had 16 rows of the gate and the same 16 of the other half.  Where split > 1 blocks share the columns, their sums are added up.
template <bool GATED, bool SPLIT, bool F32> struct Finish {
    static constexpr int kLanes = GATED ? 16 : 32, kAtOnce = 128 / kLanes, kTurns = GATED ? 2 : 4;  // threads of a row of x; rows of x at once; turns that are fetched for together
    using Bits = FourOf<F32>;
    using One = std::conditional_t<F32, uint32_t, uint16_t>;
    const TcArgs &a;
    const float *sums;
    int64_t row;       // the thread's first output
    bool whole;        // its four lie side by side and aligned
    Bits residual[GATED ? 1 : kTurns];
    const One *ahead = nullptr;  // the next residual; columns from it on
    int left = 0;

    __device__ __forceinline__ Finish(const TcArgs &a, const float *from, int64_t r0) : a(a) {
        const int part = threadIdx.x % kLanes;
        row = r0 + 4 * part;
        whole = a.wide && row + 4 <= a.n;
        sums = from + (GATED ? 32 * (part >> 2) + 4 * (part & 3) : 4 * part);
    }
    __device__ __forceinline__ int turn() const { return (threadIdx.x & 127) / kLanes; }
    // The four at p, or those of them that there are.
    __device__ __forceinline__ Bits load(const One *p) const {
        if (whole) return *reinterpret_cast<const Bits *>(p);
        One v[4];
#pragma unroll
        for (int j = 0; j < 4; j++) v[j] = row + j < a.n ? p[j] : 0;
        Bits b;
        memcpy(&b, v, sizeof b);
        return b;
    }
    // The residuals of a thread's columns, kTurns of them on their way: begin() asks for the first, of rows of x from x0 on, and each turn for the one that takes
    // its place, below column `end`.
    __device__ __forceinline__ void begin(int64_t x0, int c, int end) {
        if constexpr (GATED) return;
        if (!a.epi.residual || row >= a.n) return;
        ahead = static_cast<const One *>(a.epi.residual) + (x0 + c) * a.epi.residual_row + row;
        left = end - c;
#pragma unroll
        for (int i = 0; i < kTurns; i++) next(i);
    }
    __device__ __forceinline__ void next(int i) {
        if (left > 0) residual[GATED ? 0 : i] = load(ahead);
        ahead += kAtOnce * a.epi.residual_row;
        left -= kAtOnce;
    }
    // The residuals of columns below `count` come into the L2 cache while the products go on.
    __device__ __forceinline__ void announce(int64_t x0, int count) const {
        if constexpr (GATED) return;
        if (!a.epi.residual || row >= a.n) return;
        for (int c = threadIdx.x & 31; c < count && x0 + c < a.b; c += 32) {
            const One *r = static_cast<const One *>(a.epi.residual) + (x0 + c) * a.epi.residual_row + (row - 4 * (threadIdx.x % kLanes)) + 32 * (threadIdx.x / 32 % 4);
            if (row - 4 * (threadIdx.x % kLanes) + 32 * (threadIdx.x / 32 % 4) < a.n) asm volatile("prefetch.global.L2 [%0];" ::"l"(r));
        }
    }
    __device__ __forceinline__ void four(const float *at, float (&v)[4]) const {
        if (!SPLIT || a.split == 1) {
            const float4 f = *reinterpret_cast<const float4 *>(at);
            v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
            return;
        }
        v[0] = v[1] = v[2] = v[3] = 0.f;
        for (int p = 0; p < a.split; p++) {
            float4 f;
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w)
                         : "r"(of_rank(shared_at(at), p)) : "memory");
            v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
        }
    }
    template <int ACT> __device__ __forceinline__ void give_as(int64_t x0, int c, int end) {
        const bool bf16 = a.type == ECASQ_BF16;
        float bias[4] = {0.f, 0.f, 0.f, 0.f};
        if (!GATED && a.epi.bias) {
            One v[4];
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = row + j < a.n ? static_cast<const One *>(a.epi.bias)[row + j] : 0;
            Bits b;
            memcpy(&b, v, sizeof b);
            widen(b, bf16, bias);
        }
        One *y = static_cast<One *>(a.y) + (x0 + c) * a.y_row + row;
        const float *at = sums + 128 * c;
#pragma unroll
        for (int i = 0; i < kTurns; i++, c += kAtOnce, y += kAtOnce * a.y_row, at += kAtOnce * 128) {
            if (c >= end) return;
            float v[4];
            four(at, v);
            if (GATED) {
                float u[4];
                four(at + 16, u);
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = activate(v[j], ACT) * u[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = activate(v[j] + bias[j], ACT);
                if (a.epi.residual) {
                    float r[4];
                    widen(residual[GATED ? 0 : i], bf16, r);
                    next(i);
#pragma unroll
                    for (int j = 0; j < 4; j++) v[j] += r[j];
                }
            }
            Bits out;
            narrow(v, bf16, out);
            if (whole) {
                *reinterpret_cast<Bits *>(y) = out;
            } else {
                One o[4];
                memcpy(o, &out, sizeof out);
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (row + j < a.n) y[j] = o[j];
            }
        }
    }
    // The columns c, c + kAtOnce, ... below end, kTurns of them.
    __device__ __forceinline__ void give(int64_t x0, int c, int end) {
        if (row >= a.n) return;
        switch (a.epi.act) {
            case ECASQ_ACT_RELU: return give_as<ECASQ_ACT_RELU>(x0, c, end);
            case ECASQ_ACT_SILU: return give_as<ECASQ_ACT_SILU>(x0, c, end);
            case ECASQ_ACT_GELU: return give_as<ECASQ_ACT_GELU>(x0, c, end);
            case ECASQ_ACT_GELU_TANH: return give_as<ECASQ_ACT_GELU_TANH>(x0, c, end);
            default: return give_as<ECASQ_ACT_NONE>(x0, c, end);
        }
    }
};

// The same by lookups; lane: the address of the lane's copy of the first entry.  (A warp of the permutes takes 21 operations of the integer pipe for
// eight codes, which left the tensor core waiting for its levels: 558 us for 8192 x 8192 by 4096 rows, and 392 with nothing decoded.)
__device__ __forceinline__ void look_up(uint32_t w, uint32_t lane, uint32_t *to) {
#pragma unroll
    for (int j = 0; j < 4; j++) to[j] = *static_cast<const uint32_t *>(__cvta_shared_to_generic(permute(w, 0, 0x4440 | j) * 128 + lane));
}

// A cluster is `split` blocks, or a pair.  Of a block's warps, the first brings in rows of x, the second issues products, the third brings in codes, the
// fourth scales; kDecodeWarps turn codes into levels; eight take sums out, each its share of the columns.  Barriers pass stages between them; those that
// the products' issuer waits for are in the first block of a pair, which issues for both.  The issuer's warp runs together, so that addresses stay in
// uniform registers: with them in one lane's registers, 8192 x 8192 by 4096 rows took 1404 us where it then took 560 (with that, results also began to leave in
// 16-byte pieces).
template <int ND, int NH, bool GATED, int SPANS, bool F32>
__global__ void __launch_bounds__(TcShape<ND, NH, GATED, F32>::kThreads, 1) k_project_tc(const __grid_constant__ CUtensorMap xm, const __grid_constant__ CUtensorMap cm,
                                                                            const __grid_constant__ TcArgs a) {
    using Shape = TcShape<ND, NH, GATED, F32>;
    constexpr bool kPair = Shape::kPair;
    constexpr int kN = Shape::kN, kDBufs = Shape::kDBufs, kXStages = Shape::kXStages, kCodeStages = Shape::kCodeStages, kCodeBars = Shape::kCodeBars, kAStages = Shape::kAStages, kAAt = Shape::kAAt, kOwn = Shape::kOwn;
    extern __shared__ char smem_raw[];
    const uint32_t base = shared_at(smem_raw) + 1023 & ~1023u;
    char *smem = smem_raw + (base - shared_at(smem_raw));
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t rank = cluster_rank(), half = kPair ? rank & 1 : 0, leader = rank - half, size = Shape::kBlocks * a.split, share = rank / Shape::kBlocks;  // (share is 0 for pairs; where the compiler knew that, 8192 x 8192 by 4096 rows took 472 us and not 390)
    const uint32_t bars = base + Shape::kBarsAt;
    const uint32_t x_full = bars, x_empty = x_full + 8 * kXStages, c_full = x_empty + 8 * kXStages, c_empty = c_full + 8 * kCodeBars,
                   a_full = c_empty + 8 * kCodeStages, a_empty = a_full + 8 * kAStages, d_full = a_empty + 8 * kAStages, d_empty = d_full + 8 * kDBufs,
                   s_full = d_empty + 8 * kDBufs, s_empty = s_full + 8 * kScales, all_done = s_empty + 8 * kScales, sums_full = all_done + 8, sums_empty = sums_full + 8, lost_at = sums_empty + 8, tmem_at = lost_at + 4;
    uint32_t *books = reinterpret_cast<uint32_t *>(smem + Shape::kBooksAt);
    constexpr int terms = F32 ? 6 : 1;
    const int kb0 = (int)((int64_t)a.blocks * share / a.split), kb1 = (int)((int64_t)a.blocks * (share + 1) / a.split);
    const int cluster = blockIdx.x / size, clusters = gridDim.x / size;

    auto lose = [&] {
        for (uint32_t r = 0; r < size; r++) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(of_rank(lost_at, r)), "r"(1) : "memory");
    };
    auto lost = [&] {
        uint32_t v;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(lost_at) : "memory");
        return v != 0;
    };
    // A wait ends when its phase has, or with the loss of the block's work: when the limit has run out here or elsewhere in the cluster.
    auto wait_for = [&](auto look) {
        if (look()) return true;
        for (uint64_t t0 = nanoseconds(); nanoseconds() - t0 < kWaitMost;)
            for (int i = 0; i < 64; i++) {
                if (look()) return true;
                if (lost()) return false;
            }
        lose();
        return false;
    };
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_for([&] { return mbar_try(bar, parity); }); };
    auto wait_warp = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, wait(bar, parity)); };
    auto wait_cluster = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, wait_for([&] { return mbar_try<true>(bar, parity); })); };

    wait_before();
    if (tid == 0) {
        for (int i = 0; i < kXStages; i++) {
            mbar_init(x_full + 8 * i, 1);
            mbar_init(x_empty + 8 * i, 1);
        }
        for (int i = 0; i < kCodeBars; i++) mbar_init(c_full + 8 * i, 1);
        for (int i = 0; i < kCodeStages; i++) mbar_init(c_empty + 8 * i, 4);
        for (int i = 0; i < kAStages; i++) {
            mbar_init(a_full + 8 * i, 4 * Shape::kBlocks);
            mbar_init(a_empty + 8 * i, 1);
        }
        for (int i = 0; i < kDBufs; i++) {
            mbar_init(d_full + 8 * i, 1);
            mbar_init(d_empty + 8 * i, (NH == 2 ? 4 : 8) * Shape::kBlocks);
        }
        for (int i = 0; i < kScales; i++) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(s_empty + 8 * i, 8);
        }
        mbar_init(all_done, 1);
        mbar_init(sums_full, 8 * a.split);
        mbar_init(sums_empty, 8 * a.split);
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(lost_at), "r"(a.lost) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tile_map_fetch(&xm);
        tile_map_fetch(&cm);
    }
    if (F32) {  // the levels' bytes: three terms of eight bits each
        if (tid < 48) {
            const int term = tid / 16, j = tid % 16;
            uint32_t bits = 0;
            if (j < a.m) {
                float v = static_cast<const float *>(a.levels)[j];
                for (int i = 0; i <= term; i++) {
                    bits = __float_as_uint(v) >> 16;
                    v -= __uint_as_float(bits << 16);
                }
            }
            reinterpret_cast<uint8_t *>(books + 8 * term)[j] = (uint8_t)bits;
            reinterpret_cast<uint8_t *>(books + 8 * term)[16 + j] = (uint8_t)(bits >> 8);
        }
    } else {  // pairs: a warp those with one second level, a lane a copy
        const uint16_t *levels = static_cast<const uint16_t *>(a.levels);
        const uint32_t mine = (lane & 15) < a.m ? levels[lane & 15] : 0;
        for (int hi = wid; hi < 16; hi += Shape::kWarps)
#pragma unroll
            for (int lo = 0; lo < 16; lo++)
                reinterpret_cast<uint32_t *>(smem + Shape::kTableAt)[(16 * hi + lo) * 32 + lane] = __shfl_sync(0xffffffffu, mine, lo) | __shfl_sync(0xffffffffu, mine, hi) << 16;
    }
    if (wid == 3) tmem_alloc<kPair>(tmem_at);
    __syncthreads();
    cluster_barrier();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_at) : "memory");

    // Tile t: the rows of x and of the matrix, by panels of rows of x that stay in the L2 cache while all of the matrix goes by.
    auto tile_of = [&](int t) {
        const int whole = a.panel * a.w_tiles, first = t / whole * a.panel, wide = min(a.panel, a.x_tiles - first), rest = t % whole;
        return make_int2(first + rest % wide, rest / wide);
    };
    // The first row of the matrix that this block has of weight tile t: 128 rows (gated: 64 of each half) from it on.
    auto rows_at = [&](int t) { return (int64_t)t * Shape::kRows + half * (GATED ? 64 : 128); };
    const int per_tile = (kb1 - kb0) * terms;  // products' blocks of a tile

    if (wid < 4) {
        if (Shape::kUneven) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegs));
        if (lane == 0 && !a.lost) {
            if (wid == 0) {  // rows of x
                uint32_t i = 0;
                bool ok = true;
                for (int t = cluster; ok && t < a.tiles; t += clusters) {
                    const int64_t x0 = (int64_t)tile_of(t).x * kN + half * Shape::kXRows;
                    for (int v = 0; ok && v < per_tile; v++, i++) {
                        const uint32_t s = i % kXStages, to = base + s * Shape::kXStage;
                        if (!(ok = wait(x_empty + 8 * s, (i / kXStages & 1) ^ 1))) break;
                        mbar_expect(x_full + 8 * s, Shape::kXStage);
                        const int kb = kb0 + v / terms;
                        const int64_t from = x0 + (terms > 1 ? kXTerm[v % terms] * a.b : 0);
#pragma unroll
                        for (int h = 0; h < NH; h++)
#pragma unroll
                            for (int q = 0; q < 2; q++)
                                tile_load(to + (2 * h + q) * (Shape::kXRows * 128), &xm, kb * 128 + 64 * q, (int32_t)(from + h * ND), x_full + 8 * s);
                    }
                }
                const uint64_t t0 = nanoseconds();
                for (uint32_t j = i > kXStages ? i - kXStages : 0; j < i; j++)  // none is on its way when the block ends
                    mbar_drain(x_full + 8 * (j % kXStages), j / kXStages & 1, t0);
            } else if (wid == 2) {  // codes
                uint32_t i = 0;
                bool ok = true;
                for (int t = cluster; ok && t < a.tiles; t += clusters) {
                    const int64_t r0 = rows_at(tile_of(t).y);
                    for (int v = 0; ok && v < per_tile; v++, i++) {
                        const uint32_t s = i % kCodeStages, to = base + kXStages * Shape::kXStage + s * kCodeStage, full = c_full + 8 * (i % kCodeBars);
                        if (!(ok = wait(c_empty + 8 * s, (i / kCodeStages & 1) ^ 1))) break;
                        mbar_expect(full, kCodeStage);
                        const int kb = kb0 + v / terms;
                        tile_load(to, &cm, kb * 64, (int32_t)r0, full);
                        tile_load(to + kCodeStage / 2, &cm, kb * 64, (int32_t)(r0 + (GATED ? a.second : 64)), full);
                    }
                }
                const uint64_t t0 = nanoseconds();
                for (uint32_t j = i > kCodeStages ? i - kCodeStages : 0; j < i; j++) mbar_drain(c_full + 8 * (j % kCodeBars), j / kCodeBars & 1, t0);
            }
        }
        if (wid == 3) {
            // Scales: of each span its groups' scales of the block's 128 rows, four a lane, as fp32.  They come kScaleLag spans ahead, the four bytes
            // that hold each.  Spans are span_blocks, or what of them is this block's; or 64 or 32 columns; of fp32 for each term.
            struct Span {
                int group, word, left, term;  // its first word of 32 columns; words that its group still has; fp32: the term
            };
            const int scale_size = a.scale_type == ECASQ_F32 ? 4 : 2, group_words = a.group / 32, last_group = (int)((a.k - 1) / a.group);
            auto advance = [&](Span &s) {
                constexpr int kWords = 4 / SPANS;
                int by = SPANS == 1 && !F32 ? 4 * a.span_blocks - (s.word & (4 * a.span_blocks - 1)) : kWords;  // (span_blocks: a power of two)
                if (F32 && (s.word + by) % 4 == 0) {
                    if (++s.term < terms) by -= 4;  // the block again
                    else s.term = 0;
                }
                s.word += by;
                s.left -= by;
                while (F32 && s.left > group_words) {
                    s.left -= group_words;
                    s.group--;
                }
                if (s.left <= 0) {
                    s.left += group_words;
                    s.group++;
                }
            };
            uint32_t asked = 0, given = 0;
            bool ok = !a.lost;
            const uint32_t to = base + Shape::kScalesAt + 4 * lane;
            for (int t = cluster; ok && t < a.tiles; t += clusters) {
                const char *from[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int64_t row = rows_at(tile_of(t).y) + (GATED ? 16 * i + (lane & 15) : 32 * i + lane);
                    from[i] = static_cast<const char *>(a.scales) + (min(row, a.n - 1) + (GATED && (lane & 16) ? a.second : 0)) * a.scale_row * scale_size;
                }
                Span ask{4 * kb0 / group_words, 4 * kb0, group_words - 4 * kb0 % group_words, 0}, give = ask;
                for (int turn = 0; ok && give.word < 4 * kb1; turn++) {
                    if (ask.word < 4 * kb1) {
                        const uint32_t slot = asked % kScales;
                        if (!(ok = wait_warp(s_empty + 8 * slot, (asked / kScales & 1) ^ 1))) break;
                        const int64_t at = (int64_t)min(ask.group, last_group) * scale_size;
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + slot * 512 + 128 * i), "l"((uintptr_t)(from[i] + at) & ~(uintptr_t)3) : "memory");
                        advance(ask);
                        asked++;
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    if (turn < kScaleLag) continue;
                    asm volatile("cp.async.wait_group %0;" ::"n"(kScaleLag) : "memory");
                    const uint32_t slot = given % kScales;
                    if (scale_size == 2) {
                        uint32_t *v = reinterpret_cast<uint32_t *>(smem + Shape::kScalesAt) + slot * 128 + lane;
                        const int64_t at = (int64_t)min(give.group, last_group) * 2;
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const uint16_t half = (uint16_t)((uintptr_t)(from[i] + at) & 2 ? v[32 * i] >> 16 : v[32 * i]);
                            v[32 * i] = __float_as_uint(a.scale_type == ECASQ_F16 ? to_f32(reinterpret_cast<const __half &>(half)) : to_f32(reinterpret_cast<const __nv_bfloat16 &>(half)));
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive_own(s_full + 8 * slot);
                    advance(give);
                    given++;
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        if (wid == 1 && rank == leader) {  // products: the whole warp, so that addresses stay in uniform registers
            const uint32_t kind = mma_kind(a.type != ECASQ_F16, 128 * Shape::kBlocks, ND);
            uint32_t xs = 0, as = 0, a_parity = 0, buf = 0, d_parity = 1;
            bool ok = !a.lost;
            // Waits for the block's levels (with BLOCK; they and the rows of x come together), and, with `fresh`, for the next NH buffers for sums: one wait
            // for all, as each costs this warp about a hundred clocks, of the thousand that the tensor core takes for a block.
            uint32_t d[NH], full[NH];
            auto ready = [&](auto block, bool fresh) {
                uint32_t empty[NH], parity[NH];
                if (fresh) {
#pragma unroll
                    for (int h = 0; h < NH; h++) {
                        d[h] = tmem + buf * ND;
                        full[h] = d_full + 8 * buf;
                        empty[h] = d_empty + 8 * buf;
                        parity[h] = d_parity;
                        buf = buf + 1 == kDBufs ? 0 : buf + 1;
                        d_parity ^= buf == 0;
                    }
                }
                const bool there = __all_sync(0xffffffffu, wait_for([&] {
                    bool r = true;
                    if (block) r = mbar_try(a_full + 8 * as + 8, a_parity);  // (the second half's levels come after the first's)
                    if (fresh) {
#pragma unroll
                        for (int h = 0; h < NH; h++) r &= mbar_try(empty[h], parity[h]);
                    }
                    return r;
                }));
                tmem_fence_after();
                return there;
            };
            for (int t = cluster; ok && t < a.tiles; t += clusters) {
                int in_span = kb0 % a.span_blocks, term = 0;
                bool fresh = true;
                for (int v = 0; v < per_tile; v++) {
                    const uint32_t x = mma_rows(base + xs * Shape::kXStage), levels_at = tmem + kAAt + as * kACols;
                    // The products of 16 entries number k0 .. k1 of the block with half h of the rows of x.
                    auto steps = [&](int h, int k0, int k1, bool add) {
#pragma unroll
                        for (int kk = k0; kk < k1; kk++)
                            mma<kPair>(d[h], levels_at + kk * 8, x + ((2 * h + kk / 4) * (Shape::kXRows * 128) + kk % 4 * 32) / 16, kind, add || kk > k0);
                    };
                    if constexpr (SPANS == 1) {
                        const bool last = F32 || v + 1 == per_tile || in_span + 1 == a.span_blocks;  // (fp32: every term's sums)
                        if (!(ok = ready(std::true_type{}, fresh))) break;
                        if (one_lane()) {
                            if (NH == 2) {
                                steps(0, 0, 8, !fresh);
                                if (last) mma_commit<kPair>(full[0], rank);
                            }
                            steps(NH - 1, 0, 4, !fresh);
                            mma_commit<kPair>(a_empty + 8 * as, rank);
                            steps(NH - 1, 4, 8, true);
                            if (last) mma_commit<kPair>(full[NH - 1], rank);
                            mma_commit<kPair>(a_empty + 8 * as + 8, rank);
                            mma_commit<kPair>(x_empty + 8 * xs, rank);
                        }
                        fresh = last;
                    } else {
#pragma unroll
                        for (int sub = 0; sub < SPANS; sub++) {
                            if (!(ok = sub ? ready(std::false_type{}, true) : ready(std::true_type{}, true))) break;
                            if (one_lane()) {
#pragma unroll
                                for (int h = 0; h < NH; h++) {
                                    steps(h, sub * (8 / SPANS), (sub + 1) * (8 / SPANS), false);
                                    mma_commit<kPair>(full[h], rank);
                                }
                                if ((sub + 1) % (SPANS / 2) == 0) mma_commit<kPair>(a_empty + 8 * (as + sub / (SPANS / 2)), rank);
                                if (sub == SPANS - 1) mma_commit<kPair>(x_empty + 8 * xs, rank);
                            }
                        }
                        if (!ok) break;
                    }
                    if (++term == terms) {
                        term = 0;
                        if (++in_span == a.span_blocks) in_span = 0;
                    }
                    xs = xs + 1 == kXStages ? 0 : xs + 1;
                    as = as + 2 == kAStages ? 0 : as + 2;
                    a_parity ^= as == 0;
                }
            }
        }
        __syncwarp();
    } else if (wid < 4 + Shape::kDecodeWarps) {
        if (Shape::kUneven) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kDecodeRegs));
        // Row of the block's 128: of a gated matrix the lower half of each warp has rows of the gate.
        const int row = 32 * (wid & 3) + lane, from = GATED ? (lane & 16) * 4 + 16 * (wid & 3) + (lane & 15) : row;
        const uint32_t there = kPair ? of_rank(a_full, leader) : a_full, swizzle = (uint32_t)(from >> 1 & 3);
        constexpr int kTeams = Shape::kTeams;  // of four warps, which take turns at the blocks
        const int team = (wid - 4) / 4;
        const int64_t total = a.tiles > cluster ? (int64_t)((a.tiles - cluster + clusters - 1) / clusters) * per_tile : 0;  // blocks of all tiles
        const char *codes = smem + kXStages * Shape::kXStage + from * 64;
        uint32_t w[16], cs = team, cb = team, c_parity = 0, xs = team, x_parity = 0, as = 2 * team, a_parity = 1, term = team % terms;
        auto step = [](uint32_t &at, uint32_t by, uint32_t stages, uint32_t &parity) {
            at += by;
            if (at >= stages) {
                at -= stages;
                parity ^= 1;
            }
        };
        // The next block's words, in the order of their columns.
        auto fetch = [&] {
            if (!wait_warp(c_full + 8 * cb, c_parity)) return false;
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const uint4 four = *reinterpret_cast<const uint4 *>(codes + cs * kCodeStage + ((q ^ swizzle) << 4));
                w[q] = four.x, w[q + 4] = four.y, w[q + 8] = four.z, w[q + 12] = four.w;
            }
            // The stage is free for other codes once these have arrived in registers: the arrival's address waits for them.  (Loads of shared memory may be
            // moved behind an arrival that does not; block 3's codes then took the place of block 0's.)
            __syncwarp();
            if (lane == 0) mbar_arrive_own(c_empty + 8 * cs + ((w[0] ^ w[1] ^ w[2] ^ w[3]) & a.none));
            cs = cs + kTeams >= kCodeStages ? cs + kTeams - kCodeStages : cs + kTeams;
            step(cb, kTeams, kCodeBars, c_parity);
            return true;
        };
        auto decode_half = [&](int half, uint32_t (&pairs)[32]) {
            if (F32) {
                uint32_t book[8];
                const uint4 *from = reinterpret_cast<const uint4 *>(books + 8 * kLevelTerm[term]);
                *reinterpret_cast<uint4 *>(book) = from[0];
                *reinterpret_cast<uint4 *>(book + 4) = from[1];
#pragma unroll
                for (int q = 0; q < 8; q++) decode(w[8 * half + q], book, pairs + 4 * q);
            } else {
#pragma unroll
                for (int q = 0; q < 8; q++) look_up(w[8 * half + q], base + Shape::kTableAt + 4 * lane, pairs + 4 * q);
            }
        };
        auto store = [&](int hb, const uint32_t (&pairs)[32]) {
            const bool free = wait_warp(a_empty + 8 * (as + hb), a_parity);
            tmem_fence_after();
            tmem_store(tmem + ((uint32_t)(wid & 3) << 21) + kAAt + (as + hb) * kACols, pairs);
            return free;
        };
        auto stored = [&](int hb) {
            tmem_stored();
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at<kPair>(there + 8 * (as + hb));
        };
        // While a half's levels are on their way to tensor memory, the next half's are looked up.
        bool ok = !a.lost && (team >= total || fetch());
        for (int64_t i = team; ok && i < total; i += kTeams) {
            uint32_t pairs[32];
            decode_half(0, pairs);
            if (!(ok = store(0, pairs))) break;
            decode_half(1, pairs);
            // One warp's word stands for the block's rows of x too, so that the issuer has one barrier to wait for.
            if ((wid & 3) == 0 && !(ok = wait_warp(x_full + 8 * xs, x_parity))) break;
            stored(0);
            if (!(ok = store(1, pairs))) break;
            if (i + kTeams < total && !(ok = fetch())) break;
            stored(1);
            step(xs, kTeams, kXStages, x_parity);
            step(as, 2 * kTeams, kAStages, a_parity);
            term = (term + kTeams) % terms;
        }
    } else {
        if (Shape::kUneven) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kAddRegs));
        const int part = (wid - 4 - Shape::kDecodeWarps) / 4, quarter = wid & 3;
        const uint32_t there = kPair ? of_rank(d_empty, leader) : d_empty, column = tmem + ((uint32_t)quarter << 21) + (NH == 2 ? 0 : part * kOwn);
        // Spans of a tile.
        const int spans = SPANS == 1 && !F32 ? (kb1 - 1) / a.span_blocks - kb0 / a.span_blocks + 1 : per_tile * SPANS;
        uint32_t buf = NH == 2 ? part : 0, d_parity = 0, turn = 0, span = 0;
        bool ok = !a.lost;
        for (int t = cluster; t < a.tiles; t += clusters, turn++) {
            const int64_t r0 = rows_at(tile_of(t).y);
            float *sums = reinterpret_cast<float *>(smem + Shape::kSumsAt) + part * Shape::kOut * 128;
            Finish<GATED, NH == 1, F32>(a, sums, r0).announce((int64_t)tile_of(t).x * kN + part * kOwn, kOwn);
            uint64_t acc[kOwn / 2];  // pairs of columns
#pragma unroll
            for (int c = 0; c < kOwn / 2; c++) acc[c] = 0;
            auto add_span = [&] {
                const uint32_t slot = 8 * (span % kScales), parity = span / kScales & 1;
                ok = __all_sync(0xffffffffu, wait_for([&] {
                    const bool there = mbar_try(s_full + slot, parity);
                    return (bool)(mbar_try(d_full + 8 * buf, d_parity) & there);
                }));
                if (!ok) return;
                const uint32_t bits = reinterpret_cast<const uint32_t *>(smem + Shape::kScalesAt)[16 * slot + 32 * quarter + lane];
                const uint64_t s = bits | (uint64_t)bits << 32;
                tmem_fence_after();
                // Sixteen columns are on their way while the sixteen before them are added: a load takes about ninety clocks until its values are there,
                // whatever its width.
                constexpr int kChunk = kOwn < 32 ? kOwn / 2 : 16;
                uint32_t d[2][kChunk];
                tmem_load<kChunk>(d[0], column + buf * ND);
                tmem_load<kChunk>(d[1], column + buf * ND + kChunk);
#pragma unroll
                for (int c = 0; c < kOwn; c += 2 * kChunk) {
                    tmem_loaded(d[0], d[1]);
                    if (c + 2 * kChunk == kOwn) {
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_at<kPair>(there + 8 * buf);
                    }
#pragma unroll
                    for (int half = 0; half < 2; half++) {
#pragma unroll
                        for (int j = 0; j < kChunk / 2; j++) {
                            uint64_t &to = acc[(c + half * kChunk) / 2 + j];
                            to = fma_pair(s, d[half][2 * j] | (uint64_t)d[half][2 * j + 1] << 32, to);
                        }
                        if (c + 2 * kChunk < kOwn) tmem_load<kChunk>(d[half], column + buf * ND + c + (2 + half) * kChunk);
                    }
                }
                span++;
                __syncwarp();
                if (lane == 0) mbar_arrive_own(s_empty + slot + (bits & a.none));
                buf += NH;
                if (buf >= kDBufs) {
                    buf -= kDBufs;
                    d_parity ^= 1;
                }
            };
            for (int j = 0; ok && j < spans; j++) add_span();
            constexpr int kOut = Shape::kOut;
            auto four_warps = [&] {
                if (part) asm volatile("bar.sync 2, 128;" ::: "memory");
                else asm volatile("bar.sync 1, 128;" ::: "memory");
            };
            int c0 = 0, c1 = kOut;
            if (NH == 1 && a.split > 1) {  // each block finishes a share of the columns, of which it adds up all blocks' sums
                ok = ok && wait_cluster(sums_empty, (turn & 1) ^ 1);
                c0 = (int)share * kOut / a.split;
                c1 = (int)(share + 1) * kOut / a.split;
            }
            Finish<GATED, NH == 1, F32> finish(a, sums, r0);
            constexpr int kTurns = finish.kTurns, kAtOnce = finish.kAtOnce;
            const int64_t first_x = (int64_t)tile_of(t).x * kN + part * kOwn;
            finish.begin(first_x, c0 + finish.turn(), (int)min((int64_t)(NH == 2 ? kOwn : c1), a.b - first_x));
#pragma unroll 1
            for (int q = 0; q < kOwn / kOut; q++) {
                const int64_t x0 = first_x + q * kOut;
                const int end = (int)min((int64_t)c1, a.b - x0);
                four_warps();
#pragma unroll
                for (int c = 0; c < kOut; c += 2) {
                    uint64_t v = acc[c / 2];
#pragma unroll
                    for (int p = 1; p < kOwn / kOut; p++) v = q == p ? acc[(p * kOut + c) / 2] : v;
                    // (A lost tile's results are NaN, and those of the tiles after it.)
                    sums[128 * c + 32 * quarter + lane] = ok ? __uint_as_float((uint32_t)v) : CUDART_NAN_F;
                    sums[128 * c + 128 + 32 * quarter + lane] = ok ? __uint_as_float((uint32_t)(v >> 32)) : CUDART_NAN_F;
                }
                if (NH == 1 && a.split > 1) {
                    __syncwarp();
                    if (ok && lane < a.split) mbar_arrive<true>(of_rank(sums_full, lane));
                    if (!(ok = ok && wait_cluster(sums_full, turn & 1)))
                        for (int c = 0; c < kOut; c++) sums[128 * c + 32 * quarter + lane] = CUDART_NAN_F;
                }
                four_warps();
                for (int c = c0 + finish.turn(); c < end; c += kTurns * kAtOnce) finish.give(x0, c, end);
            }
            if (NH == 1 && a.split > 1) {
                __syncwarp();
                if (ok && lane < a.split) mbar_arrive<true>(of_rank(sums_empty, lane));
            }
        }
        if (!ok && lane == 0 && a.status) atomicOr(a.status, ECASQ_BAD_WAIT);
    }
    // A block ends when the products that read its memory, and the arrivals that they send, are through.
    __syncthreads();
    if (wid == 1 && lane == 0) {
        if (rank == leader) mma_commit<kPair>(all_done, rank);
        mbar_drain(all_done, 0, nanoseconds());
    }
    __syncthreads();
    cluster_barrier();
    if (wid == 3) tmem_free<kPair>(tmem);
}

// Clusters of `size` blocks that the card holds at once, asked once a device.
template <typename K> static int tc_held(K *kernel, int size, int threads, int smem, std::atomic<int> *known, int *held) {
    int device = 0;
    ECASQ_CUDA_TRY(cudaGetDevice(&device));
    *held = device < kDevices ? known[device].load(std::memory_order_acquire) : 0;
    if (*held > 0) return ECASQ_OK;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)size);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ECASQ_CUDA_TRY(cudaOccupancyMaxActiveClusters(held, kernel, &cfg));
    if (*held < 1) return ECASQ_ECUDA;
    if (device < kDevices) known[device].store(*held, std::memory_order_release);
    return ECASQ_OK;
}

template <int ND, int NH, bool GATED, int SPANS, bool F32> static int launch_tc(const CUtensorMap &xm, const CUtensorMap &cm, const TcArgs &a, cudaStream_t st) {
    using Shape = TcShape<ND, NH, GATED, F32>;
    static_assert(Shape::kBytes <= 227 * 1024 && Shape::kBytes > 114 * 1024, "one block an SM: tensor memory is the block's alone");
    static std::atomic<int> allowed[kDevices], known[kSplitMost + 1][kDevices];
    auto *kernel = k_project_tc<ND, NH, GATED, SPANS, F32>;
    const int size = Shape::kBlocks * a.split;
    int rc = allow_smem(kernel, Shape::kBytes, allowed), held = 0;
    if (!rc) rc = tc_held(kernel, size, Shape::kThreads, Shape::kBytes, known[a.split], &held);
    if (rc) return rc;
    return launch_clusters(kernel, dim3((unsigned)(std::min(a.tiles, held) * size)), dim3((unsigned)size), Shape::kThreads, Shape::kBytes, st, xm, cm, a);
}
template <int ND, int NH, bool GATED> static int launch_tc_spans(const CUtensorMap &xm, const CUtensorMap &cm, const TcArgs &a, cudaStream_t st) {
    if (a.type == ECASQ_F32) {
        if (a.group % 128 == 0) return launch_tc<ND, NH, GATED, 1, true>(xm, cm, a, st);
        if (a.group % 64 == 0) return launch_tc<ND, NH, GATED, 2, true>(xm, cm, a, st);
        return launch_tc<ND, NH, GATED, 4, true>(xm, cm, a, st);
    }
    if (a.group % 128 == 0) return launch_tc<ND, NH, GATED, 1, false>(xm, cm, a, st);
    if (a.group % 64 == 0) return launch_tc<ND, NH, GATED, 2, false>(xm, cm, a, st);
    return launch_tc<ND, NH, GATED, 4, false>(xm, cm, a, st);
}

// By the widths of a tile that launch_project_tc chooses among.
template <bool GATED> static int launch_tc_width(int width, const CUtensorMap &xm, const CUtensorMap &cm, const TcArgs &a, cudaStream_t st) {
    switch (width) {
        case 32: return launch_tc_spans<32, 1, GATED>(xm, cm, a, st);
        case 64: return launch_tc_spans<64, 1, GATED>(xm, cm, a, st);
        case 128: return launch_tc_spans<128, 1, GATED>(xm, cm, a, st);
        default: return launch_tc_spans<128, 2, GATED>(xm, cm, a, st);
    }
}
int launch_tc_gated(int width, const CUtensorMap &xm, const CUtensorMap &cm, const TcArgs &a, cudaStream_t st);

}  // namespace ecasq
