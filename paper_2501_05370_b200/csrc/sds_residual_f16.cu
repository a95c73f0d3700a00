// The residual norm's kernels for a stream of f16 and a branch of f16 (one source per pair of types: they compile side by side).
#include "sds_residual.cuh"

namespace sds {

cudaError_t residual_f16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  return residual_launch<F16, F16>(a, vec, backward, st);
}

}  // namespace sds
