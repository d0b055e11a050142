// matvec_gated.cu -- the kernels of ecasq_gated for 16-bit types and few rows of x.
#include "matvec16.cuh"

namespace ecasq {

int launch_matvec_gated(MatvecArgs &a, int32_t type, bool scales32, int32_t group, cudaStream_t st) { return launch_matvec_types<kGated>(a, type, scales32, group, st); }

}  // namespace ecasq
