// Host-side facts about the current device that the stand-alone entry points need.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace efcp {

constexpr int kMaxKnownDevices = 64;

// SM count of the current device, -1 when there is none.  The attribute is asked for once per
// device; the answer cannot change.
inline int device_sms() {
  static std::atomic<int> known[kMaxKnownDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxKnownDevices) {
    (void)cudaGetLastError();
    return -1;
  }
  int n = known[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    return -1;
  }
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace efcp
