// attend_coded8.cu -- ecasq_attend's kernels for rows coded with eight levels.
#include "attend.cuh"

namespace ecasq {
int launch_attend_coded8(AttendArgs &a, bool bf16, int64_t b, cudaStream_t st) {
    return bf16 ? launch_attend_heads<__nv_bfloat16, 8>(a, b, st) : launch_attend_heads<__half, 8>(a, b, st);
}
}  // namespace ecasq
