// The residual norm's kernels for a stream of floats and a branch of floats (one source per pair of types: they compile side by side).
#include "sds_residual.cuh"

namespace sds {

cudaError_t residual_f32(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  return residual_launch<float, float>(a, vec, backward, st);
}

}  // namespace sds
