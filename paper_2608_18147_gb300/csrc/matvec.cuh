// matvec.cuh -- what the kernels of ecasq_matvec share.
//
// y = x W^T for W of 4-bit codes.  A byte of codes is two weights, and one lookup in a table of all 256 pairs of levels, in
// shared memory, gives both.  The packed order of the codes (ecasq_pack) lets a lane (g, t) = (lane / 4, lane mod 4) read
// 16 bytes of row g of a 128-column block, the words t, t + 4, t + 8 and t + 12, so that one step of all lanes covers 32
// neighbouring columns, which lie in one scale group; the scale is applied to the fp32 sums of its group.
#pragma once

#include <algorithm>

#include "epilogue.cuh"

namespace ecasq {

struct MatvecArgs {
    const void *x, *levels, *scales;
    const uint8_t *codes;
    void *y;
    int32_t *status;
    int64_t x_row, code_row, scale_row, y_row, n, k;
    int32_t b, m, groups;
    int32_t warps_k;              // warps that share a row tile along k, a power of two; the others take other tiles
    int32_t chunk;                // columns that one pass over the rows covers, a multiple of 128
    int32_t slices, slice;        // 16-bit types: blocks of a cluster that share a run of rows, and their columns each, a multiple of 128
    bool keep;                    // 16-bit types: sums of rows are kept for another pass or slice
    int32_t stages;               // stages of the codes' ring
    int32_t pitch, scale_pitch;   // 16-bit types: bytes from one row to the next in a stage, and among the scales
    int32_t pieces_below;         // 16-bit types: halves of stages that lie below the table
    uint32_t lost;                // test hook: 1 where blocks begin as if a wait had run out
    int64_t second;               // gated: rows of the matrix before its other half
    Epilogue epi;                 // what follows the product
    uint32_t div_mul, div_shift;  // words of 32 columns to scale groups: w div (group / 32), as umulhi(w, div_mul) >> div_shift
                                  // or w >> div_shift if div_mul is 0
};

constexpr int kWarps = 16, kThreads = 32 * kWarps;  // a block is alone on its SM
constexpr int kRowsMost = 512, kRowSumBytes = kRowsMost * 8 * 4;  // rows of a block; their sums where several passes add up
constexpr int kSpins = 1 << 18;                     // of a wait, each of some microseconds: about two seconds

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t to, const void *from, int bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < kSpins; i++) {
        uint32_t done;
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done) : "r"(bar), "r"(parity), "r"(1000) : "memory");
        if (done) return true;
    }
    return false;
}
// Waits that run out.  A word of shared memory holds 0, or 1 more than the round of the pass in which a wait ran out: written
// before the round's barrier, read behind it.  (A thread that is a round ahead may have written already; `round` tells.)
__device__ __forceinline__ void set_word(uint32_t at, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t get_word(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ bool lost_by(uint32_t at, int round) { return get_word(at) - 1 <= (uint32_t)round; }
// Before a block whose wait ran out ends, it waits, with the limit again, for the copies that are still on their way, so that none writes
// to its shared memory when that is another's.  Bit s of `parity` is that of the next wait for stage s.  Those of the rounds
// after `round`, which has stage s, that were asked for:
__device__ __forceinline__ void drain_ahead(uint32_t bars, uint32_t &parity, int s, int round, int rounds, int stages) {
    for (int i = 1; i < stages && round + i < rounds; i++) {
        s = s + 1 == stages ? 0 : s + 1;
        bar_wait(bars + 8 * s, parity >> s & 1);
        parity ^= 1u << s;
    }
}
// and those of every stage that have been waited for.
__device__ __forceinline__ void drain_lost(uint32_t bars, uint32_t parity, int stages) {
    for (int s = 0; s < stages; s++) bar_wait(bars + 8 * s, ~parity >> s & 1);
}

// The scale group of word w (32 columns each).
__device__ __forceinline__ uint32_t group_of(const MatvecArgs &a, uint32_t w) {
    w = a.div_mul ? __umulhi(w, a.div_mul) >> a.div_shift : w >> a.div_shift;
    return min(w, (uint32_t)a.groups - 1);
}

// Blocks of a launch, one for each SM (152), more where a block would have over `most` rows.  The block's run of rows:
// whole eights, as even as they can be.
static inline int64_t row_blocks(int64_t n, int most) { return std::max(std::min<int64_t>(cdiv(n, 8), 152), cdiv(cdiv(n, 8), most / 8)); }
__device__ __forceinline__ int64_t row_of(const MatvecArgs &a, unsigned block, unsigned blocks) { return min(a.n, (a.n + 7) / 8 * block / blocks * 8); }

// What follows a product's sum v: nothing, ecasq_project's epilogue, or with u, that of the same row of the other half, ecasq_gated's.
enum After { kPlain, kProject, kGated };
template <typename T, After AFTER> __device__ __forceinline__ T result(const MatvecArgs &a, float v, float u, float bias, float residual) {
    if (AFTER == kProject) v = activate(v + bias, a.epi.act) + residual;
    if (AFTER == kGated) v = activate(v, a.epi.act) * u;
    return from_f32<T>(v);
}
// What ecasq_project adds to output r of row i of x.
template <typename T, After AFTER> __device__ __forceinline__ float bias_of(const MatvecArgs &a, int64_t r) {
    return AFTER == kProject && a.epi.bias ? to_f32(static_cast<const T *>(a.epi.bias)[r]) : 0.f;
}
template <typename T, After AFTER> __device__ __forceinline__ float residual_of(const MatvecArgs &a, int64_t i, int64_t r) {
    return AFTER == kProject && a.epi.residual ? to_f32(static_cast<const T *>(a.epi.residual)[i * a.epi.residual_row + r]) : 0.f;
}

// The kernels' launches, a unit each: fp32 and 16-bit types; a.n is the number of outputs.
int launch_matvec_f32(MatvecArgs &a, After after, int32_t group, cudaStream_t st);
int launch_matvec_project(MatvecArgs &a, int32_t type, bool scales32, int32_t group, cudaStream_t st);
int launch_matvec_gated(MatvecArgs &a, int32_t type, bool scales32, int32_t group, cudaStream_t st);

}  // namespace ecasq
