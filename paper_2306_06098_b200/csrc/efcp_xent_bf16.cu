// The linear cross-entropy kernels for bf16 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_bf16(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st) {
  return xent_gemm<__nv_bfloat16>(mode, p, blocks, st);
}
cudaError_t xent_prepare_bf16(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<__nv_bfloat16>(p, backward, sms, st);
}

}  // namespace efcp
