// codes.cuh -- element types and checks shared by the operators on 4-bit codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <utility>

#include "common.cuh"

namespace ecasq {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

static inline bool type_ok(int32_t t) { return t == ECASQ_F32 || t == ECASQ_F16 || t == ECASQ_BF16; }
static inline int64_t type_size(int32_t t) { return t == ECASQ_F32 ? 4 : 2; }
static inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// t div n for 0 <= t < 2^31: umulhi(t, mul) >> shift, or t >> shift if mul is 0.  With 2^(c-1) < n < 2^c the
// quotient is floor(t ceil(2^(31+c) / n) / 2^(31+c)): the rounding up adds less than t / 2^(31+c) < 2^-c < 1 / n (Granlund
// and Montgomery 1994).
struct FastDiv {
    uint32_t mul = 0, shift = 0;
    explicit FastDiv(int32_t n) {
        int c = 0;
        while (((int64_t)1 << c) < n) c++;
        if (((int64_t)1 << c) == n) {
            shift = (uint32_t)c;
        } else {
            mul = (uint32_t)((((uint64_t)1 << (31 + c)) + n - 1) / n);
            shift = (uint32_t)(c - 1);
        }
    }
};

// Lets a kernel have `bytes` of dynamic shared memory, once for each device: done[device] says so.
constexpr int kDevices = 16;
template <typename K> static inline int allow_smem(K *kernel, int bytes, std::atomic<int> *done) {
    int device = 0;
    ECASQ_CUDA_TRY(cudaGetDevice(&device));
    if (device < kDevices && done[device].load(std::memory_order_acquire)) return ECASQ_OK;
    ECASQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (device < kDevices) done[device].store(1, std::memory_order_release);
    return ECASQ_OK;
}

// Launches a kernel whose first statement is wait_before(): its blocks may be placed while the kernel before it in the stream still
// runs.  (In a row of calls: a product with 1024 x 1024 codes 3.5 us, and 3.9 launched after the kernel before it has ended;
// attention over 64 sequences of 100 keys 9.8 and 10.2 us; 32 x 8 cache rows 2.4 and 2.7 us.)
template <typename... P, typename... A>
static inline int launch_clusters(void (*kernel)(P...), dim3 grid, dim3 cluster, int threads, int smem, cudaStream_t st, A &&...args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster.x;
    attr[1].val.clusterDim.y = cluster.y;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster.x * cluster.y > 1 ? 2 : 1;
    note_launch();
    ECASQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...));
    return ECASQ_OK;
}
template <typename... P, typename... A>
static inline int launch_early(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t st, A &&...args) {
    return launch_clusters(kernel, grid, dim3(1), threads, smem, st, std::forward<A>(args)...);
}
// Waits until the kernel before this one has ended and what it wrote can be read, then lets the blocks of the kernel after this one
// be placed as soon as all of this one's have been.  Every block does so before it reads or writes memory, and before it ends, so
// that the kernel after this one has waited for all that came before.
__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory"); }

// What a cluster's threads wrote to shared memory before it can be read by all of them after it.  (Threads that have ended do not count.)
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// The address in the cluster of what lies at `at` in the shared memory of block `rank`.
__device__ __forceinline__ uint32_t of_rank(uint32_t at, uint32_t rank) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    return there;
}

// The limits that ecasq_cache_t states; bytes of a row's entries and of its codebook.
static inline bool cache_ok(const ecasq_cache_t *c) {
    if (!c || !c->rows || !type_ok(c->type) || c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->d < 1 || c->d > 256)
        return false;
    if (c->pages > INT64_MAX / c->page_size) return false;
    const int64_t e = c->levels_n ? 1 : type_size(c->type);
    if (!aligned16(c->rows) || c->row_page * e % 16 || c->row_slot * e % 16 || c->row_head * e % 16) return false;
    if (!c->levels_n) return c->d * e % 16 == 0;
    if ((c->levels_n != 8 && c->levels_n != 16) || c->type == ECASQ_F32 || c->d % 32 || !c->levels) return false;
    return aligned16(c->levels) && c->level_page % 8 == 0 && c->level_slot % 8 == 0 && c->level_head % 8 == 0;
}

}  // namespace ecasq
