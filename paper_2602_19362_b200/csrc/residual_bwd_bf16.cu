// The kernels of the residual norm's gradient for rows of bf16.
#include "residual_host.cuh"

namespace oapl {

int residual_bwd_bf16(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  return route_residual_level<__nv_bfloat16, false>(p, level, arrays, n_sm, run, st);
}

}  // namespace oapl
