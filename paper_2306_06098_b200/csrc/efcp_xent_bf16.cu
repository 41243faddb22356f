// The linear cross-entropy kernels for bf16 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_bf16(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st) {
  return backward ? xent_launch<__nv_bfloat16, true>(p, pairs, st) : xent_launch<__nv_bfloat16, false>(p, pairs, st);
}
cudaError_t xent_prepare_bf16(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<__nv_bfloat16>(p, backward, sms, st);
}
cudaError_t xent_finish_bf16(const XentPrep& p, int sms, cudaStream_t st) { return xent_finish<__nv_bfloat16>(p, sms, st); }

}  // namespace efcp
