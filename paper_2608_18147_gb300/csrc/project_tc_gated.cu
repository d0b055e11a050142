// project_tc_gated.cu -- the tensor-core kernels of ecasq_gated.
#include "project_tc.cuh"

namespace ecasq {

int launch_tc_gated(int width, const CUtensorMap &xm, const CUtensorMap &cm, const TcArgs &a, cudaStream_t st) { return launch_tc_width<true>(width, xm, cm, a, st); }

}  // namespace ecasq
