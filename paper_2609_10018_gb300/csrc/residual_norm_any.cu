// The form of the kernel of residual_norm.cuh for rows of any alignment and number of columns (a file of its own, since
// the two forms' variants take half a minute each to compile).
#include "residual_norm.cuh"

namespace elasto {

cudaError_t residual_norm_any_launch(const elasto_residual_norm_args& u, int* status, cudaStream_t s) {
  return residual::launch<false>(u, status, s);
}

}  // namespace elasto
