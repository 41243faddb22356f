// Host side of the group-norm calls (include/efcp.h): argument checks, and how the work is
// cut into tiles, chunks and clusters.  The kernels are in efcp_gn.cuh.
#include "efcp.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "efcp_device.h"
#include "efcp_gn.h"

namespace efcp {
namespace {

constexpr int kTypeBytes[3] = {4, 2, 2};
constexpr int kStreamedBlocksPerSM = 4;
constexpr int kMaxRowsPerThread = 64;  // keeps a thread's sums short: see Stats in efcp_gn.cuh

bool valid(const efcp_group_norm* d) {
  if (!d || d->n < 0 || d->rows < 1 || d->channels < 1 || d->groups < 1) return false;
  if (d->channels >= (1ll << 30) || d->channels % d->groups) return false;
  if (d->dtype < 0 || d->dtype > 2 || d->param_dtype < 0 || d->param_dtype > 2) return false;
  if (d->act < 0 || d->act > EFCP_ACT_SILU) return false;
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return false;
  const int64_t most = 1ll << 40;
  if (d->rows > most / d->channels || (d->n && d->rows * d->channels > most / d->n)) return false;
  return true;
}

// Rows and samples of a tensor: strides that keep every offset in 63 bits, rows apart; for an
// output also samples apart (in either order: rows inside samples or samples inside rows).
bool valid_strides(const efcp_group_norm* d, int64_t batch, int64_t row, bool output) {
  const int64_t most = 1ll << 50;
  if (row < d->channels || batch < 0 || row > most / d->rows) return false;
  if (d->n > 1 && batch > most / d->n) return false;
  if (output && d->n > 1) {
    const bool rows_inside = batch >= (d->rows - 1) * row + d->channels;
    const bool samples_inside =
        batch >= d->channels && (d->rows == 1 || row >= (d->n - 1) * batch + d->channels);
    if (!rows_inside && !samples_inside) return false;
  }
  return true;
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Tensor {
  const void* ptr;
  int64_t batch, row;
};

// The widest of 16 bytes, 4 bytes and one element that every address is a multiple of and whole
// groups can be cut into.
int pick_vec(const efcp_group_norm& d, const Tensor* t, int nt) {
  const int size = kTypeBytes[d.dtype], per = int(d.channels / d.groups);
  for (int bytes : {16, 4}) {
    const int w = bytes / size;
    if (w == 1) continue;
    bool ok = d.channels % w == 0;
    for (int i = 0; i < nt; ++i)
      ok = ok && reinterpret_cast<uintptr_t>(t[i].ptr) % bytes == 0 && t[i].row % w == 0 &&
           t[i].batch % w == 0;
    const int unit = w / gcd(per, w);  // groups whose channels are a whole number of accesses
    if (ok && (unit == 1 || int64_t(unit) * per / w <= kGnThreads)) return w;
  }
  return 1;
}

int floor_log2(int64_t v) {
  int n = 0;
  while ((2ll << n) <= v) ++n;
  return n;
}

// How `threads` threads lie over rows of the tile's channels.  Where a row has a power of two of
// accesses, up to 32, the lanes of a warp that share a channel add up by shuffles.  (Filling other rows up to
// a power of two with idle threads was slower: 65 us against 56 us for 8 x 64 x 64 x 320 fp32 backward.)
void set_layout(int threads, int vec, Gn* p) {
  const int64_t width = int64_t(p->tile_groups) * p->per;
  p->cols = int(std::min<int64_t>(threads, width / vec));
  p->pitch_log = -1;
  if (p->cols <= 32 && (p->cols & (p->cols - 1)) == 0) p->pitch_log = floor_log2(p->cols);
  p->lanes_rows = threads / p->cols;
  p->lanes_rows_log = floor_log2(p->lanes_rows);
  p->fold = gcd(p->per, vec);
  p->folded_cols = p->cols * (vec / p->fold);
  p->folded_per = std::min(p->per / p->fold, p->folded_cols);
  p->lanes_log = std::min(5, floor_log2(std::max(1, threads / p->tile_groups)));
  p->val_rows = p->pitch_log >= 0 ? threads / 32 : p->lanes_rows;
  p->val_floats = (p->val_rows * p->cols * vec + 3) / 4 * 4;
}

// Tiles of at most `groups` groups and not much less than half of that, a multiple of `unit` and all of
// nearly the same size: those that leave the fewest threads without work (65 columns on 128 threads would
// leave half of them).
void set_tiles(const efcp_group_norm& d, int vec, int unit, int64_t groups, Gn* p) {
  const int64_t most = std::max<int64_t>(1, groups / unit);
  double best = 0;
  for (int64_t k = most; k >= (most + 1) / 2; --k) {
    int64_t tiles = ceil_div(d.groups, k * unit);
    const int64_t size = ceil_div(ceil_div(d.groups, tiles), unit) * unit;
    tiles = ceil_div(d.groups, size);
    const int64_t cols = std::min<int64_t>(kGnThreads, size * p->per / vec);
    const double use = double(kGnThreads / cols) / double(tiles);
    if (use > best * 1.001) {
      best = use;
      p->tiles = int(tiles);
      p->tile_groups = int(size);
    }
  }
}

// Whether a sample's tile fits on chip; then tiles, the cluster's size and the shared memory of a
// block.  Narrow tiles come first, as they need smaller clusters: 64 bytes a row with 16-byte accesses
// (256 x 28 x 28 x 128 bf16 forward 27 us against 29 us with 128), 128 with narrower ones
// (200 x 30 x 30 x 37 forward 16 us against 21 us with 64), 32 where nothing else fits; of equal tiles
// clusters of 8 blocks before larger ones, and four blocks per SM before two.  (Tiles of 32 bytes in clusters of
// 8 before wider ones in up to 16: 128 x 90 x 90 x 64 fp16 forward 77 us against 70, 64 x 60 x 60 x 128 fp32
// backward 114 against 105, but 200 x 50 x 50 x 37 bf16 forward 49 against 74.)  Where a sample has few rows the tiles
// are wider, up to 16 rows for a thread forward, 8 backward, as long as there are three tiles per SM
// (1000 x 1 x 1 x 768 bf16 forward 9.6 us against 46 us, 256 x 7 x 7 x 512 bf16 backward 18 us against 47;
// with 16 rows backward 256 x 14 x 14 x 256 43 us against 37).  Tiles
// too few to occupy the GPU in clusters of eight are made narrower, down to 16 bytes (3 x 37 x 53 x 120 fp16
// of 2-byte accesses backward 9.7 us against 13.5; with a limit twice as high 4 x 32 x 32 x 128 fp32 forward
// 5.3 us against 4.9), and a GPU still not filled gets larger clusters, as long as a thread keeps two rows.
bool plan_resident(const efcp_group_norm& d, int vec, bool backward, int sms, Gn* p,
                   size_t* smem) {
  const int size = kTypeBytes[d.dtype], per = p->per, unit = vec / gcd(per, vec);
  if (int64_t(unit) * per / vec > kGnThreads) return false;
  const int64_t widest = int64_t(kGnThreads) * vec / per;  // groups a block is wide enough for
  const int64_t row = gn_resident_row_bytes(vec, size, backward);
  struct Try {
    int64_t bytes, smem, most;
  };
  int64_t wide = vec * size == 16 ? 64 : 128;
  if (d.n > 0) {
    const int64_t deep = ceil_div(int64_t(kGnThreads) * (backward ? 8 : 16) * vec * size, d.rows);
    wide = std::max(wide, std::min(deep, d.channels * size / ceil_div(3 * sms, d.n)));
  }
  while (wide > 16 && d.n * ceil_div(d.channels * size, wide) * 16 < 3 * sms) wide /= 2;
  for (const Try t : {Try{wide, kGnSmemOf4, 8}, Try{wide, kGnSmemOf4, 16}, Try{32, kGnSmemOf4, 16},
                      Try{wide, kGnSmemOf2, 16}, Try{32, kGnSmemOf2, 16}}) {
    const int64_t groups = std::max<int64_t>(1, ceil_div(t.bytes / size, per));
    set_tiles(d, vec, unit, std::min(ceil_div(groups, unit) * unit, widest), p);
    set_layout(kGnThreads, vec, p);
    const int64_t fixed = gn_resident_fixed_bytes(p->val_floats, p->tile_groups,
                                                  p->tile_groups * per, backward);
    const int64_t deep = std::min<int64_t>((t.smem - fixed) / row, kMaxRowsPerThread);
    if (deep < 1) continue;
    int64_t blocks = ceil_div(d.rows, p->lanes_rows * deep);
    if (blocks > t.most) continue;
    const int64_t items = std::max<int64_t>(1, d.n * p->tiles);
    if (items * blocks < 2 * sms && blocks < 8) {
      const int64_t fill = std::min<int64_t>(8, ceil_div(2 * sms, items));
      blocks = std::max(blocks, std::min(fill, d.rows / (2 * p->lanes_rows)));
    }
    p->chunk_rows = ceil_div(d.rows, blocks);
    p->chunks = int(blocks);
    p->thread_rows = int(ceil_div(p->chunk_rows, p->lanes_rows));
    p->links_log = floor_log2(blocks) + ((1 << floor_log2(blocks)) < blocks);
    *smem = size_t(fixed + p->thread_rows * row);
    return true;
  }
  return false;
}

// The widest tiles, and as many chunks as fill the GPU, with no thread taking more than
// kMaxRowsPerThread rows.
void plan_streamed(const efcp_group_norm& d, int vec, int sms, Gn* p) {
  const int per = p->per, unit = vec / gcd(per, vec);
  set_tiles(d, vec, unit, std::max<int64_t>(1, int64_t(kGnThreads) * vec / per), p);
  set_layout(kGnThreads, vec, p);
  const int64_t lanes_rows = p->lanes_rows;
  const int64_t rounds = ceil_div(int64_t(p->tile_groups) * per / vec, p->cols);
  const int64_t items = std::max<int64_t>(1, d.n * p->tiles);
  int64_t chunks = ceil_div(int64_t(sms) * kStreamedBlocksPerSM, items);
  chunks = std::min(chunks, ceil_div(d.rows, lanes_rows));
  const int64_t longest = std::max<int64_t>(1, kMaxRowsPerThread / rounds) * lanes_rows;
  chunks = std::max(chunks, ceil_div(d.rows, longest));
  p->chunk_rows = ceil_div(d.rows, chunks);
  p->chunks = int(ceil_div(d.rows, p->chunk_rows));
}

struct Plan {
  Gn gn;
  GnLaunch launch;
  int64_t part, total;  // floats of the workspace
};

int make_plan(const efcp_group_norm& d, const Tensor* t, int nt, bool backward, int sms,
              Plan* out) {
  Gn& p = out->gn;
  p = Gn{};
  p.n = d.n;
  p.rows = d.rows;
  p.channels = int(d.channels);
  p.groups = d.groups;
  p.per = int(d.channels / d.groups);
  p.param_dtype = d.param_dtype;
  p.eps = d.eps;
  p.inv_rows = 1.0 / double(d.rows);
  p.inv_total = float(1.0 / (double(d.rows) * double(p.per)));
  p.x_batch = d.x_batch; p.x_row = d.x_row;
  p.y_batch = d.y_batch; p.y_row = d.y_row;
  p.dy_batch = d.dy_batch; p.dy_row = d.dy_row;
  GnLaunch& l = out->launch;
  l.vec = pick_vec(d, t, nt);
  l.act = d.act;
  l.backward = backward;
  l.resident = plan_resident(d, l.vec, backward, sms, &p, &l.smem);
  if (!l.resident) plan_streamed(d, l.vec, sms, &p);
  const int64_t blocks = d.n * p.tiles * p.chunks;
  const int64_t joins = d.n * ceil_div(backward ? d.channels : d.groups, 32);
  if (blocks >= (1ll << 31) || joins >= (1ll << 31) || d.n * d.groups >= (1ll << 33))
    return EFCP_ETOOBIG;
  l.blocks = unsigned(blocks);
  out->part = out->total = 0;
  if (backward) {
    out->part = (l.resident ? d.n : d.n * p.chunks) * 2 * d.channels;
    out->total = l.resident ? 0 : d.n * 2 * d.channels;
  } else if (!l.resident) {
    out->part = d.n * p.chunks * 3 * d.groups;
  }
  return EFCP_OK;
}

int run(Plan& plan, int dtype, cudaStream_t st) {
  plan.launch.st = st;
  const cudaError_t e = dtype == EFCP_F32    ? gn_launch_f32(plan.gn, plan.launch)
                        : dtype == EFCP_BF16 ? gn_launch_bf16(plan.gn, plan.launch)
                                             : gn_launch_f16(plan.gn, plan.launch);
  if (e == cudaSuccess) return EFCP_OK;
  (void)cudaGetLastError();
  return EFCP_ECUDA;
}

bool misaligned(const void* p, int bytes) {
  return !p || reinterpret_cast<uintptr_t>(p) % unsigned(bytes) != 0;
}

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

// How the work is cut depends on the alignment of the tensors, which is not known here: the
// largest of the possible needs.
int64_t efcp_group_norm_workspace_bytes(const efcp_group_norm* desc, int32_t backward) {
  if (!valid(desc)) return -1;
  int sms = device_sms();
  if (sms < 1) sms = 148;  // no device: the SM count of a B200
  int64_t most = 0;
  for (uintptr_t align : {16, 4, 2}) {
    Plan plan;
    const Tensor t{reinterpret_cast<const void*>(align), 0, 0};
    if (make_plan(*desc, &t, 1, backward != 0, sms, &plan) == EFCP_OK)
      most = std::max(most, plan.part + plan.total);
  }
  return std::max<int64_t>(16, most * 4);
}

int efcp_group_norm_forward(const efcp_group_norm* desc, const void* x, const void* weight,
                            const void* bias, void* y, float* mean, float* rstd, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || !valid_strides(desc, desc->x_batch, desc->x_row, false) ||
      !valid_strides(desc, desc->y_batch, desc->y_row, true))
    return EFCP_EINVAL;
  if (desc->n == 0) return EFCP_OK;
  const int size = kTypeBytes[desc->dtype], psize = kTypeBytes[desc->param_dtype];
  if (misaligned(x, size) || misaligned(y, size) || misaligned(mean, 4) || misaligned(rstd, 4) ||
      misaligned(workspace, 16) || (weight && misaligned(weight, psize)) ||
      (bias && misaligned(bias, psize)))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Plan plan;
  const Tensor t[2] = {{x, desc->x_batch, desc->x_row}, {y, desc->y_batch, desc->y_row}};
  const int rc = make_plan(*desc, t, 2, false, sms, &plan);
  if (rc != EFCP_OK) return rc;
  if (workspace_bytes < plan.part * 4) return EFCP_ENOMEM;
  Gn& p = plan.gn;
  p.x = x; p.y = y; p.weight = weight; p.bias = bias;
  p.mean = mean; p.rstd = rstd; p.part = static_cast<float*>(workspace);
  return run(plan, desc->dtype, static_cast<cudaStream_t>(stream));
}

int efcp_group_norm_backward(const efcp_group_norm* desc, const void* dy, const void* x,
                             const float* mean, const float* rstd, const void* weight,
                             const void* bias, void* dx, void* dweight, void* dbias,
                             void* workspace, int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || !valid_strides(desc, desc->x_batch, desc->x_row, false) ||
      !valid_strides(desc, desc->dy_batch, desc->dy_row, false) ||
      !valid_strides(desc, desc->y_batch, desc->y_row, true))
    return EFCP_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int size = kTypeBytes[desc->dtype], psize = kTypeBytes[desc->param_dtype];
  if ((weight && misaligned(weight, psize)) || (bias && misaligned(bias, psize)) ||
      (dweight && misaligned(dweight, psize)) || (dbias && misaligned(dbias, psize)))
    return EFCP_EINVAL;
  if (desc->n == 0) {
    for (void* out : {dweight, dbias})
      if (out && cudaMemsetAsync(out, 0, size_t(desc->channels) * psize, st) != cudaSuccess)
        return EFCP_ECUDA;
    return EFCP_OK;
  }
  if (misaligned(x, size) || misaligned(dy, size) || misaligned(dx, size) ||
      misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(workspace, 16))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Plan plan;
  const Tensor t[3] = {{x, desc->x_batch, desc->x_row},
                       {dy, desc->dy_batch, desc->dy_row},
                       {dx, desc->y_batch, desc->y_row}};
  const int rc = make_plan(*desc, t, 3, true, sms, &plan);
  if (rc != EFCP_OK) return rc;
  if (workspace_bytes < (plan.part + plan.total) * 4) return EFCP_ENOMEM;
  Gn& p = plan.gn;
  p.x = x; p.dy = dy; p.y = dx; p.weight = weight; p.bias = bias;
  p.mean = const_cast<float*>(mean); p.rstd = const_cast<float*>(rstd);
  p.part = static_cast<float*>(workspace);
  p.total = p.part + plan.part;
  p.dweight = dweight; p.dbias = dbias;
  return run(plan, desc->dtype, st);
}

}  // extern "C"
