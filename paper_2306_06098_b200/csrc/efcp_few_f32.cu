// The linear cross entropy of a few tokens for fp32 operands.
#include "efcp_xent_few.cuh"

namespace efcp {

cudaError_t few_launch_f32(const XentFew& p, bool vec, bool backward, cudaStream_t st) {
  return few_launch<float>(p, vec, backward, st);
}

}  // namespace efcp
