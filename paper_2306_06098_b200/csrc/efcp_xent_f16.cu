// The linear cross-entropy kernels for f16 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_f16(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st) {
  return xent_gemm<__half>(mode, p, blocks, st);
}
cudaError_t xent_prepare_f16(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<__half>(p, backward, sms, st);
}

}  // namespace efcp
