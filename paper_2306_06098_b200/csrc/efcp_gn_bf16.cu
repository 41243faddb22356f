// Group norm on bfloat16 tensors.
#include "efcp_gn.cuh"

namespace efcp {

cudaError_t gn_launch_bf16(const Gn& p, const GnLaunch& l) {
  if (l.vec == 8) return launch_vec<__nv_bfloat16, 8>(p, l);
  return l.vec == 2 ? launch_vec<__nv_bfloat16, 2>(p, l) : launch_vec<__nv_bfloat16, 1>(p, l);
}

}  // namespace efcp
