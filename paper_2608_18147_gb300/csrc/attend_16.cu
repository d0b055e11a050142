// attend_16.cu -- ecasq_attend's kernels for plain 16-bit rows.
#include "attend.cuh"

namespace ecasq {
int launch_attend_16(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st) {
    return bf16 ? launch_attend_heads<__nv_bfloat16, 0>(a, b, st) : launch_attend_heads<__half, 0>(a, b, st);
}
}  // namespace ecasq
