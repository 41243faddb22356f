// The RMS-norm and dropout kernels for bf16 elements.
#include "efcp_rms.cuh"

namespace efcp {

cudaError_t rms_launch_bf16(const Rms& p, const RmsLaunch& l) { return rms_launch<__nv_bfloat16>(p, l); }

}  // namespace efcp
