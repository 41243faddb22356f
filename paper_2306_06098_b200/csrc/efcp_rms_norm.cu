// Host side of the RMS-norm and dropout calls (include/efcp.h): argument checks, and how rows are shared out.
// The kernels are in efcp_rms.cuh.
#include "efcp.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "efcp_device.h"
#include "efcp_rms.h"
#include "efcp_status.h"

namespace efcp {

__device__ int operators_status;

int* device_status() {
  void* p = nullptr;
  if (cudaGetSymbolAddress(&p, operators_status) == cudaSuccess) return static_cast<int*>(p);
  (void)cudaGetLastError();
  return nullptr;
}

namespace {

constexpr int kTypeBytes[3] = {4, 2, 2};
constexpr int kColumns = 256;  // of a chunk: see efcp_rows.cuh
constexpr int64_t kMostSmem = 114600;  // leaves an SM room for two blocks, with what is not dynamic
constexpr int64_t kMostBlocks = (1ll << 31) - 1;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool valid(const efcp_rms_norm* d) {
  if (!d || d->rows < 0 || d->d < 1 || d->d >= (1ll << 30)) return false;
  if (d->rows > (1ll << 40) / d->d) return false;
  if (d->dtype < 0 || d->dtype > 2 || d->param_dtype < 0 || d->param_dtype > 2) return false;
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return false;
  if (!(d->p >= 0. && d->p <= 1.)) return false;
  return d->p == 0. || reinterpret_cast<uintptr_t>(d->rng) % 8 == 0;
}

bool misaligned(const void* p, int bytes) {
  return !p || reinterpret_cast<uintptr_t>(p) % unsigned(bytes) != 0;
}
bool maybe_misaligned(const void* p, int bytes) { return p && misaligned(p, bytes); }

// Rows of an input: one behind the other in either order or the same one again, offsets within 63 bits.
bool valid_row(const efcp_rms_norm* d, const void* p, int64_t row) {
  return !p || (row >= 0 && row <= (1ll << 50) / std::max<int64_t>(1, d->rows));
}

bool wide(const efcp_rms_norm* d, const void* p, int64_t row) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && row * kTypeBytes[d->dtype] % 16 == 0);
}

Drop drop_of(const efcp_rms_norm* d) {
  Drop r{};
  r.threshold = uint32_t(std::lrint(d->p * 65536.0));
  r.scale = r.threshold < 65536 ? 65536.f / float(65536 - r.threshold) : 0.f;
  r.seed = d->seed;
  r.offset = d->offset;
  // (kernels read what this points to, whether anything is dropped or not)
  r.rng = r.threshold ? reinterpret_cast<const unsigned long long*>(d->rng) : nullptr;
  return r;
}

Rms common(const efcp_rms_norm* d) {
  Rms p{};
  p.rows = d->rows;
  p.d = int(d->d);
  p.param_dtype = d->param_dtype;
  p.eps = d->eps;
  p.inv_d = float(1.0 / double(d->d));
  p.drop = drop_of(d);
  return p;
}

// Chunks that a warp keeps, warps of a row, rows of a block.  (One chunk a warp: what it holds is little, and many
// warps hide each other's waits.  Backward 1531 x 1111 fp32 13.0 us, 17.1 with four chunks a warp; forward 8.1 and 5.9.)
void share(const efcp_rms_norm* d, Rms* p, RmsLaunch* l) {
  const int64_t chunks = ceil_div(d->d, kColumns);
  if (chunks > 64) {
    l->kept = 0;
    p->warps = int(std::min<int64_t>(32, chunks));
  } else {
    l->kept = chunks <= 16 ? 1 : chunks <= 32 ? 2 : 4;
    p->warps = int(ceil_div(chunks, l->kept));
  }
  p->groups = l->kept && p->warps < 8 ? 8 / p->warps : 1;
}

// Rows through shared memory, where a group of warps has two places at least: whether that is so, and how.  Units of
// several rows for short ones.  Two places: with more bytes on their way the memory gets slower (forward 16384 x 4096
// bf16: 90 us with two, 104 with three or four).  The plain kernels take what is little (there is nothing to fetch ahead),
// and fp32 rows that begin anywhere, forward: their loads of 4 bytes are as good as any (5000 x 1111: 22.5 us, 27.9 here;
// bf16, 20000 x 1111: 61 and 53).
bool plan_ring(const efcp_rms_norm* d, RmsOp op, bool vec, int inputs, bool weight, int sms, Rms* p, RmsLaunch* l) {
  if (d->rows < 2 * sms || d->d > 8192) return false;
  const bool backward = op == kRmsBackward;
  if (!vec && !backward && d->dtype == EFCP_F32) return false;
  // groups of eight that a row touches, wherever it begins
  const int64_t eights = vec ? d->d / 8 : (d->d + 14) / 8;
  const int64_t chunks = ceil_div(eights, 32), row_bytes = d->d * kTypeBytes[d->dtype];
  if (chunks > 32 || d->rows * chunks < (vec && backward ? 16 : 64) * sms) return false;
  RmsRing& q = l->ring;
  q = RmsRing{};
  q.inputs = inputs;
  q.lanes = 32;
  while (q.lanes > 1 && eights <= q.lanes / 2) q.lanes /= 2;
  q.rows = 32 / q.lanes;
  q.reps = 1;
  while (vec && chunks == 1 && q.reps < 8 && row_bytes * q.rows * q.reps < 1024) q.reps *= 2;
  q.row_bytes = int(row_bytes);
  q.pitch = int(ceil_div(row_bytes, 16) * 16 + 16);
  // (not vec: room for the pieces of 16 bytes that rows begin and end in: see efcp_rms_ring.cuh)
  q.unit_bytes = int(vec ? row_bytes * q.rows * q.reps : 48 + q.pitch * q.rows + 64);
  const auto share = [&](int64_t kept) {
    p->warps = int(std::min<int64_t>(8, ceil_div(chunks, kept)));
    p->groups = 8 / p->warps;
    const int64_t k = ceil_div(chunks, p->warps);
    l->kept = k <= 2 ? int(k) : 4;
  };
  const bool few = d->rows * chunks < 64 * sms, quantized = op == kRmsE4M3 || op == kRmsInt8;
  share(few ? 1 : backward || d->dtype == EFCP_F32 ? 2 : 4);
  if (l->kept == 4 && !quantized && 4 * p->groups * inputs * int64_t(q.unit_bytes) > 98304) share(2);
  q.weight_at = 512;  // behind the barriers
  // two places for each group, as many groups as fit; 16 warps on an SM
  q.stages = 2;
  int64_t stage, per_sm;
  while (true) {
    const int64_t weights = vec ? d->d : p->groups * p->warps * l->kept * kColumns;  // (not vec: as each lane reads it)
    q.data_at = int(ceil_div(q.weight_at + (weight ? weights * 4 : 0), 128) * 128);
    stage = int64_t(p->groups) * inputs * q.unit_bytes;
    per_sm = std::max(2, 16 / (p->warps * p->groups));
    if (q.data_at + 2 * stage <= 2 * kMostSmem / per_sm) break;
    if (--p->groups < 1) return false;
  }
  l->ringed = true;
  // (above 48 KB by itself where it is near, so that a launch raises the kernel's limit: what is not dynamic counts too)
  l->smem = size_t(q.data_at + q.stages * stage);
  if (l->smem > 40 * 1024) l->smem = std::max<size_t>(l->smem, 48 * 1024 + 16);
  const int64_t units = ceil_div(d->rows, q.rows * q.reps);
  l->blocks = unsigned(std::min<int64_t>(per_sm * sms, ceil_div(units, p->groups)));
  // the rows of a group are a multiple of eight apart
  if (!vec)
    while (int64_t(l->blocks) * p->groups * q.rows % 8) ++l->blocks;
  l->parts = l->blocks;
  return true;
}

struct Backward {
  unsigned blocks;
  int64_t parts;
};
Backward backward_blocks(const efcp_rms_norm* d, int sms, const Rms& p, const RmsLaunch& l) {
  const int64_t rows = ceil_div(d->rows, p.groups);
  const int64_t per_sm = std::max(1, 16 / (p.groups * p.warps));
  const int64_t blocks = std::max<int64_t>(1, std::min(rows, per_sm * sms));
  if (l.kept) return {unsigned(blocks), blocks * p.groups};
  const int64_t tiles = ceil_div(d->d, kColumns);
  const int64_t y = std::max<int64_t>(1, std::min(ceil_div(d->rows, 32), ceil_div(8 * sms, tiles)));
  return {unsigned(blocks), 8 * y};
}

int run(Rms& p, RmsLaunch& l, int dtype, cudaStream_t st) {
  l.st = st;
  p.status = device_status();
  if (!p.status) return EFCP_ECUDA;
  const cudaError_t e = dtype == EFCP_F32    ? rms_launch_f32(p, l)
                        : dtype == EFCP_BF16 ? rms_launch_bf16(p, l)
                                             : rms_launch_f16(p, l);
  if (e == cudaSuccess) return EFCP_OK;
  (void)cudaGetLastError();
  return EFCP_ECUDA;
}

int forward(const efcp_rms_norm* d, RmsOp op, const void* x, int64_t x_row, const void* residual,
            int64_t residual_row, const void* weight, void* y, int out_bytes, float* scales,
            int32_t block, void* h, float* rstd, void* stream) {
  if (!valid(d) || !valid_row(d, x, x_row) || !valid_row(d, residual, residual_row))
    return EFCP_EINVAL;
  if (d->rows == 0) return EFCP_OK;
  const int size = kTypeBytes[d->dtype];
  const bool summed = residual || d->p > 0.;
  if (misaligned(x, size) || maybe_misaligned(residual, size) || misaligned(y, out_bytes) ||
      maybe_misaligned(weight, kTypeBytes[d->param_dtype]) || (summed && misaligned(h, size)) ||
      maybe_misaligned(rstd, 4))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Rms p = common(d);
  RmsLaunch l{};
  l.op = op;
  l.vec = d->d % 8 == 0 && wide(d, x, x_row) && wide(d, residual, residual_row) && wide(d, weight, 0) &&
          (!summed || wide(d, h, 0)) && reinterpret_cast<uintptr_t>(y) % 16 == 0;
  // (the 8-bit outputs take no dropout; columns that share a scale have to lie on multiples of eight)
  const bool ring = (op == kRmsForward || d->p == 0.) && (l.vec || !block) && reinterpret_cast<uintptr_t>(y) % 16 == 0 &&
                    (!summed || wide(d, h, 0));
  if (!ring || !plan_ring(d, op, l.vec, residual ? 2 : 1, weight, sms, &p, &l)) {
    share(d, &p, &l);
    const int64_t blocks = ceil_div(d->rows, p.groups);
    if (blocks > kMostBlocks) return EFCP_ETOOBIG;
    l.blocks = unsigned(blocks);
  }
  p.x = x; p.x_row = x_row; p.residual = residual; p.residual_row = residual_row;
  p.weight = weight; p.y = y; p.h = summed ? h : nullptr; p.rstd = rstd;
  p.scales = scales; p.block = block;
  p.blocks = block ? int(ceil_div(d->d, block)) : 1;
  p.block_shift = block == 128 ? 7 : block == 64 ? 6 : 5;
  p.most = op == kRmsInt8 ? 127.f : 448.f;
  return run(p, l, d->dtype, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

int efcp_rms_norm_forward(const efcp_rms_norm* desc, const void* x, int64_t x_row,
                          const void* residual, int64_t residual_row, const void* weight, void* y,
                          void* h, float* rstd, void* stream) {
  if (!valid(desc)) return EFCP_EINVAL;
  return forward(desc, kRmsForward, x, x_row, residual, residual_row, weight, y,
                 kTypeBytes[desc->dtype], nullptr, 0, h, rstd, stream);
}

int efcp_rms_norm_quantize(const efcp_rms_norm* desc, int32_t format, int32_t block, const void* x,
                           int64_t x_row, const void* residual, int64_t residual_row,
                           const void* weight, void* q, float* scales, void* h, float* rstd,
                           void* stream) {
  if (!valid(desc) || (format != EFCP_E4M3 && format != EFCP_INT8)) return EFCP_EINVAL;
  if (block != 0 && block != 32 && block != 64 && block != 128) return EFCP_EINVAL;
  if (desc->rows && misaligned(scales, 4)) return EFCP_EINVAL;
  return forward(desc, format == EFCP_E4M3 ? kRmsE4M3 : kRmsInt8, x, x_row, residual, residual_row,
                 weight, q, 1, scales, block, h, rstd, stream);
}

int64_t efcp_rms_norm_workspace_bytes(const efcp_rms_norm* desc) {
  if (!valid(desc)) return -1;
  int sms = device_sms();
  if (sms < 1) sms = 148;  // no device: the SM count of a B200
  Rms p = common(desc);
  RmsLaunch l{};
  // (whether and how the rows go through shared memory hangs on pointers that are not known here)
  int64_t parts = 0;
  for (int inputs : {2, 3})
    for (bool vec : {false, true})
      for (bool weight : {false, true})
        if ((!vec || desc->d % 8 == 0) && plan_ring(desc, kRmsBackward, vec, inputs, weight, sms, &p, &l))
          parts = std::max<int64_t>(parts, l.parts);
  share(desc, &p, &l);
  parts = std::max(parts, backward_blocks(desc, sms, p, l).parts);
  return std::max<int64_t>(16, parts * desc->d * 4);
}

int efcp_rms_norm_backward(const efcp_rms_norm* desc, const void* dy, int64_t dy_row, const void* h,
                           int64_t h_row, const void* dh, int64_t dh_row, const float* rstd,
                           const void* weight, void* dx, void* dresidual, void* dweight,
                           void* workspace, int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || !valid_row(desc, dy, dy_row) || !valid_row(desc, h, h_row) ||
      !valid_row(desc, dh, dh_row))
    return EFCP_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int size = kTypeBytes[desc->dtype], psize = kTypeBytes[desc->param_dtype];
  if (maybe_misaligned(dweight, psize) || maybe_misaligned(weight, psize)) return EFCP_EINVAL;
  if (desc->rows == 0) {
    if (dweight && cudaMemsetAsync(dweight, 0, size_t(desc->d) * psize, st) != cudaSuccess)
      return EFCP_ECUDA;
    return EFCP_OK;
  }
  if (misaligned(dy, size) || misaligned(h, size) || maybe_misaligned(dh, size) ||
      misaligned(rstd, 4) || maybe_misaligned(dx, size) || maybe_misaligned(dresidual, size) ||
      (dweight && misaligned(workspace, 16)))
    return EFCP_EINVAL;
  if (!dx && !dresidual && !dweight) return EFCP_OK;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Rms p = common(desc);
  RmsLaunch l{};
  l.op = kRmsBackward;
  l.vec = desc->d % 8 == 0 && wide(desc, dy, dy_row) && wide(desc, h, h_row) && wide(desc, dh, dh_row) &&
          wide(desc, weight, 0) && wide(desc, dx, 0) && wide(desc, dresidual, 0);
  const bool ring = wide(desc, dx, 0) && wide(desc, dresidual, 0);
  if (!ring || !plan_ring(desc, kRmsBackward, l.vec, dh ? 3 : 2, weight, sms, &p, &l)) {
    share(desc, &p, &l);
    const Backward b = backward_blocks(desc, sms, p, l);
    l.blocks = b.blocks;
    l.parts = b.parts;
  }
  if (dweight && workspace_bytes < l.parts * desc->d * 4) return EFCP_ENOMEM;
  p.dy = dy; p.dy_row = dy_row; p.x = h; p.x_row = h_row; p.dh = dh; p.dh_row = dh_row;
  p.rstd = const_cast<float*>(rstd); p.weight = weight;
  p.dx = dx; p.dresidual = dresidual; p.dweight = dweight;
  p.part = dweight ? static_cast<float*>(workspace) : nullptr;
  return run(p, l, desc->dtype, st);
}

int efcp_dropout(const efcp_rms_norm* desc, const void* x, int64_t x_row, const void* residual,
                 int64_t residual_row, void* y, void* stream) {
  if (!valid(desc) || !valid_row(desc, x, x_row) || !valid_row(desc, residual, residual_row))
    return EFCP_EINVAL;
  if (desc->rows == 0) return EFCP_OK;
  const int size = kTypeBytes[desc->dtype];
  if (misaligned(x, size) || maybe_misaligned(residual, size) || misaligned(y, size))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Rms p = common(desc);
  RmsLaunch l{};
  l.op = kDropout;
  // one row behind the other: no matter where rows begin
  l.flat = x_row == desc->d && (!residual || residual_row == desc->d) && wide(desc, x, 0) && wide(desc, residual, 0) &&
           wide(desc, y, 0);
  l.vec = desc->d % 8 == 0 && wide(desc, x, x_row) && wide(desc, residual, residual_row) && wide(desc, y, 0);
  p.warps = p.groups = 1;
  const int64_t chunks = desc->rows * ceil_div(desc->d, kColumns);
  l.blocks = unsigned(std::min<int64_t>(ceil_div(l.flat ? ceil_div(desc->rows * desc->d, kColumns) : chunks, 8), 8ll * sms));
  p.x = x; p.x_row = x_row; p.residual = residual; p.residual_row = residual_row; p.y = y;
  return run(p, l, desc->dtype, static_cast<cudaStream_t>(stream));
}

int efcp_operators_status(void) {
  int s = 0;
  if (cudaMemcpyFromSymbol(&s, operators_status, sizeof s) == cudaSuccess) return s;
  (void)cudaGetLastError();
  return EFCP_ECUDA;
}

}  // extern "C"
