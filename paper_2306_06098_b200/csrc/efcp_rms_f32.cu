// The RMS-norm and dropout kernels for f32 elements.
#include "efcp_rms.cuh"

namespace efcp {

cudaError_t rms_launch_f32(const Rms& p, const RmsLaunch& l) { return rms_launch<float>(p, l); }

}  // namespace efcp
