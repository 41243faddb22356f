// Kernels that may begin while the one before them in the stream ends: what the launch costs, and the
// start of the blocks, then lies behind that kernel's last blocks.
#pragma once

#include <cuda_runtime.h>

#include <utility>

namespace efcp {

// The kernel before in the stream has ended, and its results are visible; the one behind may begin.
// A kernel started by `launch` calls this before it touches global memory.
__device__ __forceinline__ void take_turn() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

// The largest dynamic shared memory that a launch may ask for: an SM then holds two blocks.
constexpr size_t kMaxDynamicSmem = 113 * 1024;

struct Shape {
  unsigned blocks, threads;
  size_t smem;       // dynamic shared memory
  unsigned cluster;  // blocks of a cluster, 0: none
};

// A kernel's attributes belong to the device, and other host threads may launch the same kernel with other
// shapes: they are set to the same values every time, never to this launch's own.
template <class... P, class... A>
cudaError_t launch(void (*kern)(P...), const Shape& s, cudaStream_t st, A&&... args) {
  if (s.cluster > 8) {
    const cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  if (s.smem > 48 * 1024) {
    if (s.smem > kMaxDynamicSmem) return cudaErrorInvalidValue;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               int(kMaxDynamicSmem));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = s.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(s.blocks);
  cfg.blockDim = dim3(s.threads);
  cfg.dynamicSmemBytes = s.smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = s.cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}

}  // namespace efcp
