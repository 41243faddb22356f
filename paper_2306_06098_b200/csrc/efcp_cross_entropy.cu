// Host side of the linear cross-entropy calls (include/efcp.h): argument checks, the cut of the vocabulary into
// pieces, the order of the launches; and the kernels that do not depend on the operands' type.  The products are in
// efcp_xent.cuh.
#include "efcp.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "efcp_device.h"
#include "efcp_launch.cuh"
#include "efcp_xent.h"

namespace efcp {
namespace {

constexpr unsigned kAllLanes = 0xFFFFFFFFu;

__device__ int xent_status;

// lse and loss of a token from the statistics of its logits' parts; a warp takes a token.
__global__ void __launch_bounds__(256) k_xent_join(const XentPrep p) {
  take_turn();
  const int lane = threadIdx.x & 31, count = *p.count;
  const long long warps = (long long)gridDim.x * 8;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < count; i += warps) {
    const float2* part = p.part + i * p.parts;
    float top = -INFINITY, sum = 0.f;
    for (int k = lane; k < p.parts; k += 32) top = fmaxf(top, part[k].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, o));
    for (int k = lane; k < p.parts; k += 32) sum += part[k].y * expf(part[k].x - top);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if (lane) continue;
    const float lse = top + logf(sum);
    const float loss = p.target[i] < 0 ? __int_as_float(0x7FC00000) : lse - p.target_logit[i];
    p.lse_out[p.order[i]] = lse;
    if (p.reduction) p.each[i] = loss;
    else p.losses[p.order[i]] = loss;
  }
}

// Their sum or mean, in a fixed order.
__global__ void __launch_bounds__(1024) k_xent_total(const XentPrep p) {
  take_turn();
  __shared__ double part[32];
  const int lane = threadIdx.x & 31, count = *p.count;
  double sum = 0;
  for (int i = threadIdx.x; i < count; i += 1024) sum += double(p.each[i]);
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
  if (lane == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  sum = part[lane];
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
  if (lane == 0) p.losses[0] = float(p.reduction == 1 ? sum / count : sum);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

constexpr int kTypeBytes[3] = {4, 2, 2};
constexpr int64_t kGradBytes = 256ll << 20;  // of the logits' gradient held at a time

bool valid(const efcp_cross_entropy* d) {
  if (!d || d->tokens < 0 || d->vocab < 1 || d->d < 1) return false;
  if (d->tokens >= (1ll << 30) || d->vocab >= (1ll << 30) || d->d >= (1ll << 24)) return false;
  if (d->dtype < 0 || d->dtype > 2 || d->reduction < 0 || d->reduction > 2) return false;
  if (d->tokens > (1ll << 40) / d->d || d->vocab > (1ll << 40) / d->d) return false;
  for (int64_t row : {d->hidden_row, d->weight_row})
    if (row < 0 || row > (1ll << 32)) return false;
  return true;
}

bool misaligned(const void* p, int bytes) {
  return !p || reinterpret_cast<uintptr_t>(p) % unsigned(bytes) != 0;
}

// How a call is cut, and where its scratch memory lies.
struct Plan {
  int planes;
  bool in_place;
  int64_t padded;      // tokens up to whole tiles
  int64_t packed_row;  // elements of a packed row
  int col_tiles, col_tile, parts;
  int64_t piece;       // columns of the vocabulary at a time
  int pieces;
  int d_tiles, d_tile;
  int64_t sum_row;
  // offsets
  int64_t count, scale, order, target, lse, coef, logit, each, part, hidden, weight, g, sum, bytes;
};

int tile_of(int64_t n, int* tiles) {
  *tiles = int(ceil_div(n, kXentCols));
  return int(round_up(ceil_div(n, *tiles), 64));
}

// Whether the tensor copies can read the weight where it lies.
bool in_place(const efcp_cross_entropy& d, const void* weight) {
  return d.dtype != EFCP_F32 && reinterpret_cast<uintptr_t>(weight) % 16 == 0 && d.weight_row % 8 == 0 &&
         d.weight_row >= d.d;
}

Plan make_plan(const efcp_cross_entropy& d, const void* weight, bool backward) {
  Plan p{};
  p.planes = d.dtype == EFCP_F32 ? 3 : 1;
  p.padded = round_up(std::max<int64_t>(1, d.tokens), kXentRows);
  p.packed_row = round_up(d.d, 8);
  p.col_tile = tile_of(d.vocab, &p.col_tiles);
  p.parts = 2 * p.col_tiles;
  p.d_tile = tile_of(d.d, &p.d_tiles);
  p.sum_row = round_up(d.d, 32);
  const int64_t most = std::max<int64_t>(1, kGradBytes / (2 * p.planes * p.padded * kXentCols));  // tiles
  p.pieces = int(ceil_div(ceil_div(d.vocab, kXentCols), most));
  p.piece = p.pieces == 1 ? round_up(d.vocab, 64) : round_up(ceil_div(d.vocab, p.pieces), kXentCols);
  p.pieces = int(ceil_div(d.vocab, p.piece));
  int64_t at = 0;
  const auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += round_up(bytes, 256);
    return here;
  };
  p.count = take(4);
  p.scale = take(8);
  p.order = take(4 * p.padded);
  p.target = take(4 * p.padded);
  p.logit = take(4 * p.padded);
  p.hidden = take(2 * p.planes * p.padded * p.packed_row);
  p.in_place = in_place(d, weight);
  if (!p.in_place) p.weight = take(2 * p.planes * d.vocab * p.packed_row);
  if (backward) {
    p.lse = take(4 * p.padded);
    p.coef = take(4 * p.padded);
    p.g = take(2 * p.planes * p.padded * p.piece);
    if (p.pieces > 1) p.sum = take(4 * p.padded * p.sum_row);
  } else {
    p.each = take(4 * p.padded);
    p.part = take(8 * p.padded * p.parts);
  }
  p.bytes = at;
  return p;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) !=
            cudaSuccess || q != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return EncodeTiled(nullptr);
    }
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// Planes of rows of `cols` elements of 2 bytes, copied in boxes of 64 x 64.
bool make_map(CUtensorMap* map, int dtype, const void* base, int64_t cols, int64_t rows, int64_t row,
              int planes, int64_t plane) {
  const EncodeTiled f = encoder();
  if (!f) return false;
  const cuuint64_t size[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(planes)};
  const cuuint64_t stride[2] = {cuuint64_t(row) * 2, cuuint64_t(planes > 1 ? plane : row) * 2};
  const cuuint32_t box[3] = {64, 64, 1}, step[3] = {1, 1, 1};
  return f(map, dtype == EFCP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
           const_cast<void*>(base), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Call {
  const efcp_cross_entropy& d;
  Plan plan;
  int sms;
  cudaStream_t st;
  XentPrep prep{};
  XentGemm gemm{};
  CUtensorMap hidden, weight, g;

  template <class T>
  T* at(void* ws, int64_t off) const {
    return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
  }

  bool begin(const void* h, const void* w, const int64_t* targets, void* ws) {
    const Plan& p = plan;
    prep.targets = reinterpret_cast<const long long*>(targets);
    prep.tokens = d.tokens;
    prep.ignore = d.ignore_index;
    prep.vocab = int(d.vocab);
    prep.d = int(d.d);
    prep.hidden = h;
    prep.hidden_row = d.hidden_row;
    prep.weight = p.in_place ? nullptr : w;
    prep.weight_row = d.weight_row;
    prep.hidden_packed = at<void>(ws, p.hidden);
    prep.weight_packed = at<void>(ws, p.weight);
    prep.packed_row = p.packed_row;
    prep.hidden_plane = p.padded * p.packed_row;
    prep.weight_plane = d.vocab * p.packed_row;
    prep.count = at<int>(ws, p.count);
    prep.scale = at<float>(ws, p.scale);
    prep.order = at<int>(ws, p.order);
    prep.target = at<int>(ws, p.target);
    prep.target_logit = at<float>(ws, p.logit);
    prep.parts = p.parts;
    prep.reduction = d.reduction;
    gemm.count = prep.count;
    gemm.order = prep.order;
    gemm.target = prep.target;
    gemm.scale = prep.scale;
    gemm.target_logit = prep.target_logit;
    gemm.parts = p.parts;
    gemm.vocab = prep.vocab;
    gemm.d = prep.d;
    gemm.planes = p.planes;
    void* status = nullptr;
    if (cudaGetSymbolAddress(&status, xent_status) != cudaSuccess) return false;
    gemm.status = static_cast<int*>(status);
    return make_map(&hidden, d.dtype, prep.hidden_packed, d.d, p.padded, p.packed_row, p.planes,
                    prep.hidden_plane) &&
           make_map(&weight, d.dtype, p.in_place ? w : prep.weight_packed, d.d, d.vocab,
                    p.in_place ? d.weight_row : p.packed_row, p.planes, prep.weight_plane);
  }

  bool prepare(bool backward) {
    const cudaError_t e = d.dtype == EFCP_F32    ? xent_prepare_f32(prep, backward, sms, st)
                          : d.dtype == EFCP_BF16 ? xent_prepare_bf16(prep, backward, sms, st)
                                                 : xent_prepare_f16(prep, backward, sms, st);
    return e == cudaSuccess;
  }

  bool multiply(XentMode mode, int64_t tiles) {
    const unsigned blocks = unsigned(std::max<int64_t>(1, std::min<int64_t>(tiles, sms)));
    const cudaError_t e = d.dtype == EFCP_F32    ? xent_gemm_f32(mode, gemm, blocks, st)
                          : d.dtype == EFCP_BF16 ? xent_gemm_bf16(mode, gemm, blocks, st)
                                                 : xent_gemm_f16(mode, gemm, blocks, st);
    return e == cudaSuccess;
  }

  bool logits(XentMode mode) {
    gemm.a = hidden;
    gemm.b = weight;
    gemm.row_tiles = -1;
    gemm.depth = gemm.d;
    return multiply(mode, plan.padded / kXentRows * gemm.col_tiles);
  }
};

int failed() {
  (void)cudaGetLastError();
  return EFCP_ECUDA;
}

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

int64_t efcp_cross_entropy_workspace_bytes(const efcp_cross_entropy* desc, const void* weight,
                                           int32_t backward) {
  if (!valid(desc)) return -1;
  return make_plan(*desc, weight, backward != 0).bytes;
}

int efcp_cross_entropy_forward(const efcp_cross_entropy* desc, const void* hidden, const void* weight,
                               const int64_t* targets, float* losses, float* lse, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || (desc->tokens && (misaligned(losses, 4) || misaligned(lse, 4)))) return EFCP_EINVAL;
  const int size = kTypeBytes[desc->dtype];
  if (desc->reduction && misaligned(losses, 4)) return EFCP_EINVAL;
  if (desc->tokens && (misaligned(hidden, size) || misaligned(targets, 8))) return EFCP_EINVAL;
  if (misaligned(weight, size) || misaligned(workspace, 256)) return EFCP_EINVAL;
  Call c{*desc, make_plan(*desc, weight, false)};
  if (workspace_bytes < c.plan.bytes) return EFCP_ENOMEM;
  if (desc->tokens == 0 && !desc->reduction) return EFCP_OK;
  c.sms = device_sms();
  if (c.sms < 1) return EFCP_ECUDA;
  c.st = static_cast<cudaStream_t>(stream);
  if (!c.begin(hidden, weight, targets, workspace)) return failed();
  c.prep.losses = losses;
  c.prep.lse_out = lse;
  c.prep.each = c.at<float>(workspace, c.plan.each);
  c.prep.part = c.gemm.part = c.at<float2>(workspace, c.plan.part);
  c.gemm.col_tiles = c.plan.col_tiles;
  c.gemm.col_tile = c.plan.col_tile;
  if (!c.prepare(false) || !c.logits(kXentStats) || xent_join(c.prep, c.sms, c.st) != cudaSuccess)
    return failed();
  return EFCP_OK;
}

int efcp_cross_entropy_backward(const efcp_cross_entropy* desc, const float* grad, int64_t grad_step,
                                const void* hidden, const void* weight, const int64_t* targets,
                                const float* lse, void* dhidden, void* dweight, void* workspace,
                                int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || grad_step < 0) return EFCP_EINVAL;
  const int size = kTypeBytes[desc->dtype];
  if (desc->tokens && (misaligned(hidden, size) || misaligned(targets, 8) || misaligned(lse, 4) ||
                       misaligned(grad, 4) || (dhidden && misaligned(dhidden, size))))
    return EFCP_EINVAL;
  if (misaligned(weight, size) || (dweight && misaligned(dweight, size)) || misaligned(workspace, 256))
    return EFCP_EINVAL;
  Call c{*desc, make_plan(*desc, weight, true)};
  if (workspace_bytes < c.plan.bytes) return EFCP_ENOMEM;
  c.st = static_cast<cudaStream_t>(stream);
  if (!dhidden && !dweight) return EFCP_OK;
  c.sms = device_sms();
  if (c.sms < 1) return EFCP_ECUDA;
  if (desc->tokens == 0) {
    if (dweight && cudaMemsetAsync(dweight, 0, size_t(desc->vocab * desc->d) * size, c.st) != cudaSuccess)
      return failed();
    return EFCP_OK;
  }
  if (!c.begin(hidden, weight, targets, workspace)) return failed();
  const Plan& p = c.plan;
  XentGemm& m = c.gemm;
  c.prep.grad = grad;
  c.prep.grad_step = grad_step;
  c.prep.lse_in = lse;
  c.prep.lse = c.at<float>(workspace, p.lse);
  c.prep.coef = c.at<float>(workspace, p.coef);
  c.prep.dhidden = dhidden;
  m.lse = c.prep.lse;
  m.coef = c.prep.coef;
  m.g = c.at<void>(workspace, p.g);
  m.g_row = p.piece;
  m.g_plane = p.padded * p.piece;
  m.sum = c.at<float>(workspace, p.sum);
  m.sum_row = p.sum_row;
  m.out_row = desc->d;
  m.piece = int(p.piece);
  if (!make_map(&c.g, desc->dtype, m.g, p.piece, p.padded, p.piece, p.planes, m.g_plane) ||
      !c.prepare(true))
    return failed();
  for (int k = 0; k < p.pieces; ++k) {
    m.v0 = int(k * p.piece);
    m.first = k == 0;
    m.last = k == p.pieces - 1;
    m.col_tile = tile_of(p.piece, &m.col_tiles);
    if (!c.logits(kXentGrad)) return failed();
    m.col_tiles = p.d_tiles;
    m.col_tile = p.d_tile;
    if (dhidden) {
      m.a = c.g;
      m.b = c.weight;
      m.row_tiles = -1;
      m.depth = m.piece;
      m.out = dhidden;
      m.vec_out = reinterpret_cast<uintptr_t>(dhidden) % 16 == 0 && desc->d * size % 16 == 0;
      if (!c.multiply(kXentHidden, p.padded / kXentRows * p.d_tiles)) return failed();
    }
    if (dweight) {
      m.a = c.g;
      m.b = c.hidden;
      m.row_tiles = int(ceil_div(std::min<int64_t>(p.piece, desc->vocab - m.v0), kXentRows));
      m.depth = -1;
      m.out = dweight;
      m.vec_out = reinterpret_cast<uintptr_t>(dweight) % 16 == 0 && desc->d * size % 16 == 0;
      if (!c.multiply(kXentWeight, int64_t(m.row_tiles) * p.d_tiles)) return failed();
    }
  }
  return EFCP_OK;
}

int efcp_cross_entropy_status(void) {
  int s = 0;
  if (cudaMemcpyFromSymbol(&s, xent_status, sizeof s) != cudaSuccess) return failed();
  return s;
}

}  // extern "C"

namespace efcp {

cudaError_t xent_join(const XentPrep& p, int sms, cudaStream_t st) {
  const long long rows = p.tokens / 8 + 1;
  cudaError_t e = launch(k_xent_join, Shape{unsigned(rows < 8ll * sms ? rows : 8ll * sms), 256, 0, 0}, st, p);
  if (e != cudaSuccess || !p.reduction) return e;
  return launch(k_xent_total, Shape{1, 1024, 0, 0}, st, p);
}

}  // namespace efcp
