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
#include "efcp_status.h"
#include "efcp_xent.h"

namespace efcp {
namespace {

constexpr unsigned kAllLanes = 0xFFFFFFFFu;

// lse and loss of a token from the statistics of its logits' parts (their largest values are in units of log2(e)); a
// warp takes a token.  The last steps are in 64 bits: lse is several times as large as the loss.  (The largest value is
// taken back by the factor that it has got, rounding and all: that is 1e-8 off log2(e), and the loss is what little
// lse is above the target's logit.)
__global__ void __launch_bounds__(256) k_xent_join(const XentPrep p) {
  take_turn();
  const int lane = threadIdx.x & 31, count = *p.count;
  const long long warps = (long long)gridDim.x * 8;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < count; i += warps) {
    const float2* part = p.part + i * p.parts;
    float top = -INFINITY, sum = 0.f;
    constexpr int kAhead = 4;  // loads on their way
    for (int k = lane; k < p.parts; k += 32 * kAhead) {
      float2 o[kAhead];
      float m = top;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        o[j] = k + 32 * j < p.parts ? part[k + 32 * j] : make_float2(-INFINITY, 0.f);
        m = fmaxf(m, o[j].x);
      }
      const float base = m == -INFINITY ? 0.f : m;
      sum *= exp2f(top - base);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) sum += o[j].y * exp2f(o[j].x - base);
      top = m;
    }
    float m = top;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAllLanes, m, o));
    sum *= exp2f(top - (m == -INFINITY ? 0.f : m));
    top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if (lane) continue;
    const double lse = double(top) / double(kLog2e) + log(double(sum));
    const float loss =
        p.target[i] < 0 ? __int_as_float(0x7FC00000) : float(lse - double(p.target_logit[i]));
    p.lse_out[p.order[i]] = float(lse);
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
  int64_t piece;       // columns of the vocabulary at a time
  int pieces;
  int shifts;  // how often a piece may be doubled, when few tokens count
  int col_tiles, col_tile;  // of the logits: all of them forward, a piece's backward
  int parts;
  int d_tiles, d_tile;
  int pairs;
  int64_t sum_row, sum_rows;
  // offsets
  int64_t count, scale, order, target, lse, coef, rest, place, logit, each, part, bounds, hidden, weight, g[2], sum, bytes;
};

// Whether the tensor copies can read the weight where it lies.
bool in_place(const efcp_cross_entropy& d, const void* weight) {
  return d.dtype != EFCP_F32 && reinterpret_cast<uintptr_t>(weight) % 16 == 0 && d.weight_row % 8 == 0 &&
         d.weight_row >= d.d;
}

// Tiles of equal width, a multiple of 128.
int tile_of(int64_t n, int* tiles) {
  *tiles = int(ceil_div(n, kXentCols));
  return int(round_up(ceil_div(n, *tiles), 128));
}

Plan make_plan(const efcp_cross_entropy& d, const void* weight, bool backward, int sms) {
  Plan p{};
  p.planes = d.dtype == EFCP_F32 ? 3 : 1;
  p.padded = round_up(std::max<int64_t>(1, d.tokens), kXentRows);
  p.packed_row = round_up(d.d, 8);
  p.pairs = std::max(1, sms / 2);
  p.d_tile = tile_of(d.d, &p.d_tiles);
  p.sum_row = round_up(d.d, 32);
  const int64_t most = std::max<int64_t>(1, kGradBytes / 2 / (2 * p.planes * p.padded * kXentCols));  // tiles
  p.pieces = int(ceil_div(ceil_div(d.vocab, kXentCols), most));
  p.piece = p.pieces == 1 ? round_up(d.vocab, 64) : round_up(ceil_div(d.vocab, p.pieces), kXentCols);
  p.pieces = int(ceil_div(d.vocab, p.piece));
  p.col_tile = tile_of(backward ? p.piece : d.vocab, &p.col_tiles);
  p.parts = 2 * p.col_tiles;
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
    p.rest = take(4 * p.padded);
    p.place = take(4 * p.padded);
    p.bounds = take(4 * (kXentBuckets + 1));
    for (int i = 0; i < std::min(2, p.pieces); ++i) p.g[i] = take(2 * p.planes * p.padded * p.piece);
    // how many rows count is not known here: the most that any number of them takes with its parts
    const int64_t rows = p.padded / kXentRows;
    while (p.shifts < kXentShifts && (p.piece << p.shifts) < d.vocab && (rows >> (p.shifts + 1)) > 0) ++p.shifts;
    int64_t parts = 0;
    for (int64_t r = 1; r <= std::min<int64_t>(rows, 2 * p.pairs + 1); ++r)
      parts = std::max<int64_t>(parts, r * xent_splits(int(r), p.d_tiles, int(p.piece << xent_shift(int(r), int(rows), p.shifts)),
                                                       p.pairs, p.planes > 1));
    p.sum_rows = std::max(rows, parts) * kXentRows;
    p.sum = take(4 * p.sum_rows * p.sum_row);
  } else {
    p.each = take(4 * p.padded);
    p.part = take(8 * p.padded * p.parts);
  }
  p.bytes = at;
  return p;
}

// Up to eight tokens have kernels of their own, which hold the hidden states in shared memory (two blocks on an SM): see
// efcp_xent_few.cuh.
bool few(const efcp_cross_entropy& d) {
  return d.tokens >= 1 && d.tokens <= kFewTokens && (d.tokens <= 4 ? 4 : 8) * round_up(d.d, 256) * 4 <= 110 * 1024;
}

struct FewPlan {
  int64_t logit, sums, bytes;
  int blocks, ranges;
};
FewPlan few_plan(const efcp_cross_entropy& d, bool backward, int sms) {
  FewPlan p{};
  const int64_t n = d.tokens <= 4 ? 4 : 8;
  p.blocks = int(std::min<int64_t>(2 * sms, ceil_div(d.vocab, 32)));
  p.ranges = int(std::max<int64_t>(1, std::min(2 * sms / ceil_div(d.d, 1024 / n), ceil_div(d.vocab, 32))));
  p.logit = round_up(8 * n * p.blocks, 256);
  p.sums = round_up(4 * n * d.vocab, 256);
  p.bytes = backward ? p.sums + 4 * n * p.ranges * round_up(d.d, 256) : p.logit + 256;
  return p;
}

XentFew few_call(const efcp_cross_entropy& d, const FewPlan& plan, const void* hidden, const void* weight,
                 const int64_t* targets) {
  XentFew p{};
  p.targets = reinterpret_cast<const long long*>(targets);
  p.ignore = d.ignore_index;
  p.tokens = int(d.tokens);
  p.vocab = int(d.vocab);
  p.d = int(d.d);
  p.padded = int(round_up(d.d, 256));
  p.blocks = plan.blocks;
  p.ranges = plan.ranges;
  p.reduction = d.reduction;
  p.hidden = hidden;
  p.hidden_row = d.hidden_row;
  p.weight = weight;
  p.weight_row = d.weight_row;
  return p;
}

int few_run(const efcp_cross_entropy& d, const XentFew& p, bool backward, cudaStream_t st) {
  const bool vec = d.d % 8 == 0 && reinterpret_cast<uintptr_t>(p.weight) % 16 == 0 &&
                   d.weight_row * kTypeBytes[d.dtype] % 16 == 0 && reinterpret_cast<uintptr_t>(p.dweight) % 16 == 0;
  const cudaError_t e = d.dtype == EFCP_F32    ? few_launch_f32(p, vec, backward, st)
                        : d.dtype == EFCP_BF16 ? few_launch_bf16(p, vec, backward, st)
                                               : few_launch_f16(p, vec, backward, st);
  if (e == cudaSuccess) return EFCP_OK;
  (void)cudaGetLastError();
  return EFCP_ECUDA;
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

// Planes of rows of `cols` elements, `row` elements apart, copied in boxes of `box_rows` rows of 128 (or 64) bytes.
bool make_map(CUtensorMap* map, int dtype, const void* base, int64_t cols, int64_t rows, int64_t row,
              int planes, int64_t plane, int box_rows, int box_bytes = 128) {
  const EncodeTiled f = encoder();
  if (!f) return false;
  const int size = kTypeBytes[dtype];
  const cuuint64_t sizes[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(planes)};
  const cuuint64_t stride[2] = {cuuint64_t(row) * size, cuuint64_t(planes > 1 ? plane : row) * size};
  const cuuint32_t box[3] = {cuuint32_t(box_bytes / size), cuuint32_t(box_rows), 1}, step[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype == EFCP_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == EFCP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return f(map, type, 3, const_cast<void*>(base), sizes, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
           box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Call {
  const efcp_cross_entropy& d;
  Plan plan;
  int sms;
  cudaStream_t st;
  XentPrep prep{};
  XentGemm gemm{};

  template <class T>
  T* at(void* ws, int64_t off) const {
    return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
  }

  // (fp32 operands are held as three bfloat16 ones)
  int operand_type() const { return d.dtype == EFCP_F16 ? EFCP_F16 : EFCP_BF16; }

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
    prep.d_tiles = p.d_tiles;
    prep.piece = gemm.piece = int(p.piece);
    prep.tiles = gemm.tiles = int(p.padded / kXentRows);
    prep.shifts = gemm.shifts = p.shifts;
    prep.pairs = p.pairs;
    gemm.count = prep.count;
    gemm.target = prep.target;
    gemm.scale = prep.scale;
    gemm.target_logit = prep.target_logit;
    gemm.parts = p.parts;
    gemm.vocab = prep.vocab;
    gemm.d = prep.d;
    gemm.d_tiles = p.d_tiles;
    gemm.d_tile = p.d_tile;
    gemm.col_tiles = p.col_tiles;
    gemm.col_tile = p.col_tile;
    gemm.status = device_status();
    if (!gemm.status) return false;
    const void* weight = p.in_place ? w : prep.weight_packed;
    const int64_t weight_row = p.in_place ? d.weight_row : p.packed_row;
    const int type = operand_type();
    const auto hidden_map = [&](CUtensorMap* m, int box) {
      return make_map(m, type, prep.hidden_packed, d.d, p.padded, p.packed_row, p.planes, prep.hidden_plane, box);
    };
    const auto weight_map = [&](CUtensorMap* m, int box) {
      return make_map(m, type, weight, d.d, d.vocab, weight_row, p.planes, prep.weight_plane, box);
    };
    return hidden_map(&gemm.hidden_rows, kXentRows / 2) && hidden_map(&gemm.hidden_cols, 64) &&
           weight_map(&gemm.weight_rows, p.col_tile / 2) && weight_map(&gemm.weight_cols, 64);
  }

  bool prepare(bool backward) {
    const cudaError_t e = d.dtype == EFCP_F32    ? xent_prepare_f32(prep, backward, sms, st)
                          : d.dtype == EFCP_BF16 ? xent_prepare_bf16(prep, backward, sms, st)
                                                 : xent_prepare_f16(prep, backward, sms, st);
    return e == cudaSuccess;
  }

  bool multiply(bool backward) {
    const unsigned pairs = unsigned(plan.pairs);
    const cudaError_t e = d.dtype == EFCP_F32    ? xent_gemm_f32(backward, gemm, pairs, st)
                          : d.dtype == EFCP_BF16 ? xent_gemm_bf16(backward, gemm, pairs, st)
                                                 : xent_gemm_f16(backward, gemm, pairs, st);
    return e == cudaSuccess;
  }

  bool finish() {
    const cudaError_t e = d.dtype == EFCP_F32    ? xent_finish_f32(prep, sms, st)
                          : d.dtype == EFCP_BF16 ? xent_finish_bf16(prep, sms, st)
                                                 : xent_finish_f16(prep, sms, st);
    return e == cudaSuccess;
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
  int sms = device_sms();
  if (sms < 1) sms = 148;  // (no device: a B200's)
  return few(*desc) ? few_plan(*desc, backward != 0, sms).bytes
                                   : make_plan(*desc, weight, backward != 0, sms).bytes;
}

int efcp_cross_entropy_forward(const efcp_cross_entropy* desc, const void* hidden, const void* weight,
                               const int64_t* targets, float* losses, float* lse, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || (desc->tokens && (misaligned(losses, 4) || misaligned(lse, 4)))) return EFCP_EINVAL;
  const int size = kTypeBytes[desc->dtype];
  if (desc->reduction && misaligned(losses, 4)) return EFCP_EINVAL;
  if (desc->tokens && (misaligned(hidden, size) || misaligned(targets, 8))) return EFCP_EINVAL;
  if (misaligned(weight, size) || misaligned(workspace, 256)) return EFCP_EINVAL;
  const int sms = device_sms();
  if (few(*desc)) {
    const FewPlan plan = few_plan(*desc, false, sms < 1 ? 148 : sms);
    if (workspace_bytes < plan.bytes) return EFCP_ENOMEM;
    if (sms < 1) return EFCP_ECUDA;
    XentFew p = few_call(*desc, plan, hidden, weight, targets);
    p.part = static_cast<float2*>(workspace);
    p.target_logit = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.logit);
    p.losses = losses;
    p.lse_out = lse;
    return few_run(*desc, p, false, static_cast<cudaStream_t>(stream));
  }
  Call c{*desc, make_plan(*desc, weight, false, sms < 1 ? 148 : sms), sms};
  if (workspace_bytes < c.plan.bytes) return EFCP_ENOMEM;
  if (desc->tokens == 0 && !desc->reduction) return EFCP_OK;
  if (sms < 1) return EFCP_ECUDA;
  c.st = static_cast<cudaStream_t>(stream);
  if (!c.begin(hidden, weight, targets, workspace)) return failed();
  c.prep.losses = losses;
  c.prep.lse_out = lse;
  c.prep.each = c.at<float>(workspace, c.plan.each);
  c.prep.part = c.gemm.part = c.at<float2>(workspace, c.plan.part);
  if (!c.prepare(false) || !c.multiply(false) || xent_join(c.prep, c.sms, c.st) != cudaSuccess)
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
  const int sms = device_sms();
  if (few(*desc)) {
    const FewPlan plan = few_plan(*desc, true, sms < 1 ? 148 : sms);
    if (workspace_bytes < plan.bytes) return EFCP_ENOMEM;
    if (!dhidden && !dweight) return EFCP_OK;
    if (sms < 1) return EFCP_ECUDA;
    XentFew p = few_call(*desc, plan, hidden, weight, targets);
    p.grad = grad;
    p.grad_step = grad_step;
    p.lse_in = lse;
    p.g = static_cast<float*>(workspace);
    p.sums = dhidden ? reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.sums) : nullptr;
    p.dhidden = dhidden;
    p.dweight = dweight;
    return few_run(*desc, p, true, static_cast<cudaStream_t>(stream));
  }
  Call c{*desc, make_plan(*desc, weight, true, sms < 1 ? 148 : sms), sms};
  if (workspace_bytes < c.plan.bytes) return EFCP_ENOMEM;
  c.st = static_cast<cudaStream_t>(stream);
  if (!dhidden && !dweight) return EFCP_OK;
  if (sms < 1) return EFCP_ECUDA;
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
  c.prep.rest = m.rest = p.planes == 1 ? c.at<float>(workspace, p.rest) : nullptr;
  c.prep.layer = weight;
  c.prep.place = c.at<int>(workspace, p.place);
  float* sum = c.at<float>(workspace, p.sum);
  c.prep.sum = sum;
  c.prep.sum_row = p.sum_row;
  c.prep.dhidden = dhidden;
  m.bounds = c.prep.bounds = p.planes == 1 && dweight ? c.at<int>(workspace, p.bounds) : nullptr;
  while ((desc->vocab - 1) / kXentRows >> c.prep.wide >= kXentBuckets) ++c.prep.wide;
  m.wide = c.prep.wide;
  m.lse = c.prep.lse;
  m.coef = c.prep.coef;
  m.dweight = dweight;
  m.box_dweight = dweight && reinterpret_cast<uintptr_t>(dweight) % 16 == 0 && desc->d * size % 16 == 0;
  const int type = c.operand_type();
  const int64_t plane = p.padded * p.piece;
  for (int s = 0; s <= p.shifts; ++s)
    for (int i = 0; i < 2; ++i) {
      const void* g = c.at<void>(workspace, p.g[p.pieces > 1 ? i : 0]);
      const int64_t wide = p.piece << s, rows = (p.padded / kXentRows >> s) * kXentRows;
      auto& map = m.g[s][i];
      if (!make_map(&map.rows, type, g, wide, rows, wide, p.planes, plane, kXentRows / 2) ||
          !make_map(&map.cols, type, g, wide, rows, wide, p.planes, plane, 64) ||
          !make_map(&map.out, type, g, wide, rows, wide, p.planes, plane, 32, p.planes == 1 ? 128 : 64))
        return failed();
    }
  if (!make_map(&m.sum_out, EFCP_F32, sum, p.sum_row, p.sum_rows, p.sum_row, 1, 0, 32) ||
      (m.box_dweight &&
       !make_map(&m.dweight_out, desc->dtype, dweight, desc->d, desc->vocab, desc->d, 1, 0, 32)))
    return failed();
  if (!c.prepare(true)) return failed();
  m.hidden = dhidden != nullptr;
  m.weight = dweight != nullptr;
  // (where pieces are wider than they might be, the last launches find nothing to do)
  for (m.turn = 0; m.turn <= p.pieces; ++m.turn)
    if (!c.multiply(true)) return failed();
  if (dhidden && !c.finish()) return failed();
  return EFCP_OK;
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
