// The linear cross-entropy kernels for f32 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_f32(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st) {
  return xent_gemm<float>(mode, p, blocks, st);
}
cudaError_t xent_prepare_f32(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<float>(p, backward, sms, st);
}

}  // namespace efcp
