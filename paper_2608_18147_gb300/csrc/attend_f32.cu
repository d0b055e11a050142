// attend_f32.cu -- ecasq_attend's kernels for plain fp32 rows.
#include "attend.cuh"

namespace ecasq {
int launch_attend_f32(AttendArgs &a, int64_t b, cudaStream_t st) { return launch_attend_rows<float, 0, 8>(a, b, st); }
}  // namespace ecasq
