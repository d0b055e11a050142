// attend_coded16.cu -- ecasq_attend's kernels for rows coded with sixteen levels.
#include "attend.cuh"

namespace ecasq {
int launch_attend_coded16(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st) {
    return bf16 ? launch_attend_heads<__nv_bfloat16, 16>(a, b, st) : launch_attend_heads<__half, 16>(a, b, st);
}
}  // namespace ecasq
