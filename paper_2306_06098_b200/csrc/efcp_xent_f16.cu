// The linear cross-entropy kernels for f16 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_f16(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st) {
  return backward ? xent_launch<__half, true>(p, pairs, st) : xent_launch<__half, false>(p, pairs, st);
}
cudaError_t xent_prepare_f16(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<__half>(p, backward, sms, st);
}
cudaError_t xent_finish_f16(const XentPrep& p, int sms, cudaStream_t st) { return xent_finish<__half>(p, sms, st); }

}  // namespace efcp
