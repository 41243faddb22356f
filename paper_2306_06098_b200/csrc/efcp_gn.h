// What the host hands to the group-norm kernels (efcp_gn.cuh), and their launch functions, one
// per element type (each compiled by itself).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace efcp {

// Threads of a block.  The sums between the passes cost a warp about a thousand instructions whatever
// its rows, so few threads with many rows are better than many with few: forward 256 x 56 x 56 x 64
// bf16 62 us with 256 threads, 53 us with 128.
constexpr int kGnThreads = 128;
static_assert((kGnThreads & (kGnThreads - 1)) == 0, "rows are shared out by shifts");

struct Gn {
  const void* x;
  const void* dy;
  void* y;  // backward: dx
  const void* weight;
  const void* bias;
  float* mean;
  float* rstd;
  float* part;   // sums of chunks (streamed) or of samples (resident, backward)
  float* total;  // streamed, backward: sums of samples
  void* dweight;
  void* dbias;
  long long x_batch, x_row, y_batch, y_row, dy_batch, dy_row;
  long long n, rows, chunk_rows;  // samples; rows of a sample, of a chunk
  int channels, groups, per;      // per: channels of a group
  int tile_groups, tiles;         // groups of a tile (the last tile may have fewer), tiles
  int chunks;                     // chunks of a sample; resident: the blocks of a cluster
  int thread_rows;                // resident: rows a thread has room for
  // How the threads of a block lie over rows and channels, the same for every tile (in a last,
  // smaller one some have nothing to do), and what follows from that for its sums.
  int cols;                       // accesses of a row side by side
  int pitch_log;                  // log2(cols) where cols is a power of two up to 32, else -1
  int lanes_rows, lanes_rows_log; // rows side by side (and its logarithm if pitch_log >= 0)
  int lanes_log;                  // 2^lanes_log lanes add up a group
  int fold;                       // channels of an access that always belong to one group
  int folded_cols, folded_per;    // values of a row, and of a group in it, after adding those
  int val_rows, val_floats;       // rows of partial sums in shared memory; floats of one set
  int links_log;                  // 2^links_log lanes join the blocks of a cluster
  double inv_rows;                // 1 / rows
  float inv_total;                // 1 / (rows per)
  int param_dtype;
  float eps;
};

// How the kernels are launched.
struct GnLaunch {
  int vec;        // elements per access: as many as fill 16 or 4 bytes, or 1
  int act;        // EFCP_ACT_*
  bool backward;
  bool resident;  // a cluster of `chunks` blocks holds a sample's tile
  unsigned blocks;
  size_t smem;    // resident: dynamic shared memory
  cudaStream_t st;
};

// Shared memory of a block when an SM is to hold four or two: of its 228 KB, 1 KB per block is
// the system's.
constexpr int64_t kGnSmemOf4 = 56 * 1024, kGnSmemOf2 = 113 * 1024;

// Shared memory of the kernels (the arrays at their start say what for).  Resident: what does not
// depend on the rows, and what a row of every thread takes.
constexpr int64_t gn_resident_fixed_bytes(int64_t val_floats, int tile_groups, int width,
                                          bool backward) {
  const int64_t wide = (int64_t(width) + 3) / 4 * 4, tg = (int64_t(tile_groups) + 3) / 4 * 4;
  return 4 * (backward ? 2 * val_floats + 8 * wide + 2 * tg
                       : 4 * val_floats + 3 * wide + 3 * tg);
}
constexpr int64_t gn_resident_row_bytes(int vec, int size, bool backward) {
  return int64_t(kGnThreads) * vec * size * (backward ? 2 : 1);
}
constexpr int64_t gn_streamed_floats(int64_t val_floats, bool backward) {
  return (backward ? 2 : 4) * val_floats;
}

cudaError_t gn_launch_f32(const Gn& p, const GnLaunch& l);
cudaError_t gn_launch_bf16(const Gn& p, const GnLaunch& l);
cudaError_t gn_launch_f16(const Gn& p, const GnLaunch& l);

}  // namespace efcp
