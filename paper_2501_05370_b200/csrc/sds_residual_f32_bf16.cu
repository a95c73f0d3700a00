// The residual norm's kernels for a stream of floats and a branch of bf16 (one source per pair of types: they compile side by side).
#include "sds_residual.cuh"

namespace sds {

cudaError_t residual_f32_bf16(ResidualNormArgs& a, bool vec, bool backward, cudaStream_t st) {
  return residual_launch<float, Bf16>(a, vec, backward, st);
}

}  // namespace sds
