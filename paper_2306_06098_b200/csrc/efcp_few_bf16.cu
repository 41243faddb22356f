// The linear cross entropy of a few tokens for bf16 operands.
#include "efcp_xent_few.cuh"

namespace efcp {

cudaError_t few_launch_bf16(const XentFew& p, bool vec, bool backward, cudaStream_t st) {
  return few_launch<__nv_bfloat16>(p, vec, backward, st);
}

}  // namespace efcp
