// The linear cross-entropy kernels for f32 operands.
#include "efcp_xent.cuh"

namespace efcp {

cudaError_t xent_gemm_f32(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st) {
  return backward ? xent_launch<float, true>(p, pairs, st) : xent_launch<float, false>(p, pairs, st);
}
cudaError_t xent_prepare_f32(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  return xent_prepare<float>(p, backward, sms, st);
}
cudaError_t xent_finish_f32(const XentPrep& p, int sms, cudaStream_t st) { return xent_finish<float>(p, sms, st); }

}  // namespace efcp
