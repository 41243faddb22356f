// Group norm on fp32 tensors.
#include "efcp_gn.cuh"

namespace efcp {

cudaError_t gn_launch_f32(const Gn& p, const GnLaunch& l) {
  return l.vec == 4 ? launch_vec<float, 4>(p, l) : launch_vec<float, 1>(p, l);
}

}  // namespace efcp
