// Waits that run out, on barriers that nothing completes and with no copy under way: what the library's bounded waits do then.
// Each probe is one block; results go to `out`.
#include <cuda_runtime.h>

#include "efcp_rms_ring.cuh"

namespace efcp {
namespace {

constexpr uint64_t kLimit = 1000000;  // 1 ms

// out: whether a wait for a phase that is done came through; for one that is not; whether that told the block's others
__global__ void k_wait(int* out) {
  __shared__ alignas(8) uint64_t bar[2];
  __shared__ int gave_up;
  const uint32_t done = tc::smem_of(bar), never = done + 8;
  gave_up = 0;
  tc::bar_init(done, 1);
  tc::bar_init(never, 1);
  tc::bar_init_fence();
  tc::bar_expect(done, 0);  // (an arrival)
  out[0] = tc::bar_wait(done, 0, &gave_up, kLimit);
  out[1] = tc::bar_wait(never, 0, &gave_up, kLimit);
  out[2] = gave_up;
  out[3] = tc::bar_wait(never, 0, &gave_up);  // (of the usual length: ends at once)
}

// A ring whose first wait runs out.  out: units asked for before (none: nothing is ever copied), whether the wait is lost, units
// asked for afterwards, whether the block's others were told
__global__ void k_ring(const Rms p, const RmsRing q, int* out) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int gave_up;
  auto r = ring_begin<float, 1, false>(p, q, smem, &gave_up);
  __syncthreads();
  if (threadIdx.x) return;
  r.in[0] = {static_cast<const char*>(p.x), p.x_row * 4};
  r.limit = kLimit;
  out[0] = int(r.asked);
  r.await();
  out[1] = r.lost;
  r.ask(r.first, 0);
  out[2] = int(r.asked);
  out[3] = gave_up;
  r.end();
}

// A block of two groups: one comes to its end while the other's wait is still running out.  out: the status; what the first would
// have told by itself
__global__ void k_late(int* out) {
  __shared__ alignas(8) uint64_t bar;
  __shared__ int gave_up;
  if (threadIdx.x == 0) {
    gave_up = 0;
    tc::bar_init(tc::smem_of(&bar), 1);
    tc::bar_init_fence();
    out[0] = 0;
  }
  __syncthreads();
  if (threadIdx.x == 0) out[1] = *(volatile int*)&gave_up;
  if (threadIdx.x >= 32) (void)tc::bar_wait(tc::smem_of(&bar), 0, &gave_up, kLimit);
  ring_tell(out, &gave_up);
}

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" int probe(int which, const float* x, int* out) {
  if (which == 0) {
    k_wait<<<1, 1>>>(out);
  } else if (which == 1) {
    k_late<<<1, 64>>>(out);
  } else {
    Rms p{};
    p.rows = 4;
    p.d = 256;
    p.warps = p.groups = 1;
    p.x = x;
    p.x_row = 256;
    RmsRing q{};
    q.stages = 2;
    q.inputs = q.rows = q.reps = 1;
    q.lanes = 32;
    q.row_bytes = q.unit_bytes = 1024;
    q.weight_at = q.data_at = 512;
    k_ring<<<1, 32, 512 + 2 * 1024>>>(p, q, out);
  }
  const cudaError_t e = cudaGetLastError();
  return int(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
