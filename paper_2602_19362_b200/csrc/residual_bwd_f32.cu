// The kernels of the residual norm's gradient for rows of f32.
#include "residual_host.cuh"

namespace oapl {

int residual_bwd_f32(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  return route_residual_level<float, false>(p, level, arrays, n_sm, run, st);
}

}  // namespace oapl
