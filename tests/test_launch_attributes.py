"""The launch helper's use of a kernel's attributes, compiled against a stand-in for the CUDA runtime: a kernel's limit of
dynamic shared memory belongs to the device, not to the calling thread, so one thread's launch must not take away what another
has just asked for."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_06098_b200", "csrc")

RUNTIME = r"""
#pragma once
#include <cstddef>
#include <functional>
#include <map>
#define __device__
#define __forceinline__ inline
enum cudaError_t { cudaSuccess = 0, cudaErrorInvalidValue = 1 };
using cudaStream_t = void*;
enum cudaFuncAttribute { cudaFuncAttributeMaxDynamicSharedMemorySize = 8, cudaFuncAttributeNonPortableClusterSizeAllowed = 14 };
struct dim3 { unsigned x, y, z; dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {} };
enum cudaLaunchAttributeID { cudaLaunchAttributeClusterDimension, cudaLaunchAttributeProgrammaticStreamSerialization };
struct cudaLaunchAttribute {
  cudaLaunchAttributeID id;
  union { struct { unsigned x, y, z; } clusterDim; int programmaticStreamSerializationAllowed; } val;
};
struct cudaLaunchConfig_t {
  dim3 gridDim, blockDim;
  size_t dynamicSmemBytes = 0;
  cudaStream_t stream = nullptr;
  cudaLaunchAttribute* attrs = nullptr;
  unsigned numAttrs = 0;
};
inline std::map<void*, int> limit, wide;      // what the attributes of a kernel are set to
inline std::function<void()> between;         // what another thread does after an attribute was set
inline bool busy = false;
template <class K>
cudaError_t cudaFuncSetAttribute(K* k, cudaFuncAttribute a, int v) {
  (a == cudaFuncAttributeMaxDynamicSharedMemorySize ? limit : wide)[reinterpret_cast<void*>(k)] = v;
  if (between && !busy) {
    busy = true;
    between();
    busy = false;
  }
  return cudaSuccess;
}
template <class... P, class... A>
cudaError_t cudaLaunchKernelEx(const cudaLaunchConfig_t* c, void (*k)(P...), A&&...) {
  void* key = reinterpret_cast<void*>(k);
  if (c->dynamicSmemBytes > 48 * 1024 && int(c->dynamicSmemBytes) > limit[key]) return cudaErrorInvalidValue;
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeClusterDimension && c->attrs[i].val.clusterDim.x > 8 && !wide[key])
      return cudaErrorInvalidValue;
  return cudaSuccess;
}
"""

MAIN = r"""
#include "efcp_launch.cuh"
#include <cstdio>
static void one(int) {}
static void two(int) {}
static int run(void (*k)(int), size_t smem, unsigned cluster) {
  return efcp::launch(k, efcp::Shape{100, 128, smem, cluster}, nullptr, 0);
}
int main() {
  // alone
  for (size_t s : {size_t(0), size_t(1000), size_t(48 * 1024), size_t(50 * 1024), size_t(113 * 1024)})
    for (unsigned c : {0u, 1u, 8u, 16u})
      if (run(two, s, c)) return std::printf("alone: %zu bytes, cluster %u\n", s, c), 1;
  // another thread launches the same kernel with less, or with a smaller cluster, between this one's
  // attributes and its launch
  for (size_t mine : {size_t(50 * 1024), size_t(112 * 1024), size_t(113 * 1024)}) {
    for (size_t other : {size_t(0), size_t(49 * 1024), size_t(56 * 1024)}) {
      for (unsigned c : {0u, 4u, 16u}) {
        limit.clear();
        wide.clear();
        bool failed = false;
        between = [&] { failed = failed || run(one, other, c); };
        failed = run(one, mine, 16) || failed;
        between = nullptr;
        if (failed) return std::printf("%zu bytes beside a launch of %zu\n", mine, other), 1;
      }
    }
  }
  if (!run(one, 228 * 1024, 0)) return std::printf("more than there is\n"), 1;
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
def test_a_launch_leaves_other_threads_their_shared_memory(tmp_path):
    (tmp_path / "cuda_runtime.h").write_text(RUNTIME)
    (tmp_path / "main.cpp").write_text(MAIN)
    exe = tmp_path / "launches"
    subprocess.run(["g++", "-std=c++17", "-Wno-attributes", "-I", str(tmp_path), "-I", CSRC, "-o", str(exe), str(tmp_path / "main.cpp")],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout
