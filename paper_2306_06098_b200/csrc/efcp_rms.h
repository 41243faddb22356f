// Between the host side of the RMS-norm and dropout calls (efcp_rms_norm.cu) and their kernels (efcp_rms.cuh),
// which are compiled once per element type.
#pragma once

#include <cuda_runtime.h>

#include "efcp_philox.cuh"

namespace efcp {

struct Rms {
  long long rows;
  int d;
  int warps, groups;  // warps that share a row, rows that a block takes at a time
  int param_dtype;
  float eps, inv_d;
  Drop drop;
  const void *x, *residual, *weight;  // x: h in the backward call
  const void *dy, *dh;
  long long x_row, residual_row, dy_row, dh_row;  // elements between rows; outputs lie row after row
  void *y, *h;                                    // h null: it is x
  float* rstd;
  void *dx, *dresidual, *dweight;  // null: not wanted
  float* part;                     // sums of dweight, a row of d for each slot
  float* scales;
  int block, blocks;  // columns that share a scale (0: a row), scales of a row
  int block_shift;    // log2(block)
  float most;         // largest value of the 8-bit type
  int* status;
};

// Rows that arrive in shared memory by bulk copies, some ahead of their use.  A group of warps has a ring of `stages`
// places of its own; a place holds a unit: one row, or several short ones that share a warp.
struct RmsRing {
  int stages, inputs;
  int rows, lanes;  // rows that a warp takes at once, lanes that share one (32 unless rows > 1)
  int reps;         // such sets of rows in a unit
  int row_bytes, unit_bytes;
  int pitch;               // bytes between rows of a unit in a place, where an input's rows are not side by side
  int weight_at, data_at;  // in shared memory: the weight in fp32, the rings
};

enum RmsOp { kRmsForward, kRmsE4M3, kRmsInt8, kRmsBackward, kDropout };

struct RmsLaunch {
  RmsOp op;
  bool vec;         // rows start on 16 bytes, and on multiples of eight elements of the logical order  (not so, but
                    // ringed: outputs start on 16 bytes)
  int kept;         // chunks that a warp keeps in registers: 1, 2, 4, or 0 (rows walked twice)
  unsigned blocks;
  long long parts;  // rows of `part`
  bool flat;        // dropout of rows that lie one behind the other
  bool ringed;      // see RmsRing
  RmsRing ring;
  size_t smem;
  cudaStream_t st;
};

cudaError_t rms_launch_f32(const Rms& p, const RmsLaunch& l);
cudaError_t rms_launch_bf16(const Rms& p, const RmsLaunch& l);
cudaError_t rms_launch_f16(const Rms& p, const RmsLaunch& l);

}  // namespace efcp
