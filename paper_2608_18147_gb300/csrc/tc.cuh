// tc.cuh -- the tensor core's instructions and the barriers between a block's warps and its cluster's, as the kernels use them.
#pragma once

#include <cuda.h>

#include "codes.cuh"

namespace ecasq {

__device__ __forceinline__ uint32_t shared_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// One lane of a warp that is together, the same each time; the compiler keeps what it computes in uniform registers.
__device__ __forceinline__ bool one_lane() {
    uint32_t is;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(is));
    return is;
}

// ---------------------------------------------------------------- barriers
__device__ __forceinline__ void mbar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// An arrival at a barrier of the block; one at any of the cluster (`bar`: an address in it); and the look whether a phase is over.  What they order: tensor
// memory with its fences, tiles brought in by copies, and the block's own shared memory.  The forms that order all of the cluster's
// memory (CLUSTER) wait for every store on its way and drop cached lines: with them everywhere a product took five times as long.
__device__ __forceinline__ void mbar_arrive_own(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
template <bool CLUSTER = false> __device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    if (CLUSTER) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <bool ELSEWHERE> __device__ __forceinline__ void mbar_arrive_at(uint32_t bar) {
    if (ELSEWHERE) mbar_arrive(bar);
    else mbar_arrive_own(bar);
}
template <bool CLUSTER = false> __device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    if (CLUSTER)
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}

// Nanoseconds, for the limits of waits.
__device__ __forceinline__ uint64_t nanoseconds() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
constexpr uint64_t kWaitMost = 2000000000;  // of a wait: two seconds

// Waits for a phase, until kWaitMost after t0.
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity, uint64_t t0) {
    while (!mbar_try(bar, parity) && nanoseconds() - t0 < kWaitMost) {}
}

// ---------------------------------------------------------------- tensor memory
// All 512 columns, of a block or of both blocks of a pair (PAIR); a whole warp of each calls these.
template <bool PAIR> __device__ __forceinline__ void tmem_alloc(uint32_t to) {
    if (PAIR) asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n\ttcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(to) : "memory");
    else asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n\ttcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(to) : "memory");
}
template <bool PAIR> __device__ __forceinline__ void tmem_free(uint32_t at) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 lanes of N neighbouring columns, a row of them a lane.  The registers hold them behind tmem_loaded() alone, through which they go, so that nothing
// reads them before: a copy to other registers would take what was in them.
template <int N> __device__ __forceinline__ void tmem_load(uint32_t (&v)[N], uint32_t at);
template <> __device__ __forceinline__ void tmem_load<8>(uint32_t (&v)[8], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(at) : "memory");
}
template <> __device__ __forceinline__ void tmem_load<16>(uint32_t (&v)[16], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                   "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(at) : "memory");
}
template <int N> __device__ __forceinline__ void tmem_loaded(uint32_t (&v)[N], uint32_t (&w)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; i += 8) {  // (volatile operations keep their order)
        asm volatile("" : "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])::"memory");
        asm volatile("" : "+r"(w[i]), "+r"(w[i + 1]), "+r"(w[i + 2]), "+r"(w[i + 3]), "+r"(w[i + 4]), "+r"(w[i + 5]), "+r"(w[i + 6]), "+r"(w[i + 7])::"memory");
    }
}
// c + a b for two fp32 at once, each as fmaf.
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// The other way; they can be read by others once tmem_stored() has returned.
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
                 "%30,%31,%32};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                 "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
                 "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- products
// Instruction descriptor: fp32 sums, both operands of one 16-bit type (bf16 or f16) with the summed index innermost.
__host__ __device__ constexpr uint32_t mma_kind(bool bf16, int m, int n) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
// Operand in shared memory: rows of 128 bytes, eight to a 1024-byte block in the 128-byte swizzle, blocks one after another.  The low word of its
// descriptor, to which a distance in 16 bytes can be added; the high word is the same for all.
__device__ __forceinline__ uint32_t mma_rows(uint32_t at) { return at >> 4 | 1u << 16; }
constexpr uint32_t kMmaRowsHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
// D (+)= A B^T over 16 entries of the summed index: A in tensor memory, 128 rows; B in shared memory.  For a pair of blocks (PAIR) each has its own rows of A and
// of D, and half of the rows of B.
template <bool PAIR> __device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t kind, bool add) {
    if (PAIR)
        asm volatile("{ .reg .pred p; .reg .b64 b; mov.b64 b, {%2, %5}; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], b, %3, p; }" ::"r"(d), "r"(a), "r"(b),
                     "r"(kind), "r"((uint32_t)add), "n"(kMmaRowsHigh)
                     : "memory");
    else
        asm volatile("{ .reg .pred p; .reg .b64 b; mov.b64 b, {%2, %5}; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p; }" ::"r"(d), "r"(a), "r"(b),
                     "r"(kind), "r"((uint32_t)add), "n"(kMmaRowsHigh)
                     : "memory");
}
// An arrival at this barrier, of a pair in both blocks, once all products issued before have been done; rank: the first block's.
template <bool PAIR> __device__ __forceinline__ void mma_commit(uint32_t bar, uint32_t rank) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)(3u << rank)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---------------------------------------------------------------- tiles
__device__ __forceinline__ void tile_load(uint32_t to, const CUtensorMap *map, int32_t c0, int32_t c1, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(c0), "r"(c1), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tile_map_fetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Describes a matrix [rows, cols] to tile_load: tiles of box_rows x box_cols, zeros outside the matrix.
int make_tile_map(CUtensorMap *map, CUtensorMapDataType type, const void *at, int64_t cols, int64_t rows, int64_t row_bytes, int box_cols, int box_rows,
                  CUtensorMapSwizzle swizzle);

}  // namespace ecasq
