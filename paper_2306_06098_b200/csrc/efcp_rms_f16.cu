// The RMS-norm and dropout kernels for f16 elements.
#include "efcp_rms.cuh"

namespace efcp {

cudaError_t rms_launch_f16(const Rms& p, const RmsLaunch& l) { return rms_launch<__half>(p, l); }

}  // namespace efcp
