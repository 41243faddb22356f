// Linear cross entropy of up to eight tokens (the formulas stand in include/efcp.h): the layer's weight is what there is to
// read, and its gradient to write; tiles of the tensor cores would be empty but for a few rows.
//
// The hidden states lie in shared memory in fp32.  A warp takes four rows of the weight, multiplies them with all
// tokens in fp32 (two products to an instruction), and adds up its lanes' parts so that each lane ends up with one logit.
// Backward the logits' gradient is written, a few values a row; then warps on columns of their own walk down the rows,
// out of the cache where they fit there: they hold the hidden states and their gradient in registers, and write the gradient
// of the weight.  The blocks' sums are added up in order.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_num.cuh"
#include "efcp_rows.cuh"
#include "efcp_xent.h"

namespace efcp {
namespace {

constexpr int kFewRows = 4, kFewTile = 8 * kFewRows;  // rows of the weight: of a warp, of a block

// e^x for x <= 0
__device__ __forceinline__ float few_exp(float x) { return exp2f(x * 1.4426950408889634f); }

// The tokens' hidden states in fp32, zeros for those that do not count.
template <typename T, int N>
__device__ __forceinline__ void few_hidden(const XentFew& p, float* h) {
  for (int t = 0; t < N; ++t) {
    const bool used = t < p.tokens && p.targets[t] != p.ignore;
    const T* from = static_cast<const T*>(p.hidden) + t * p.hidden_row;
    for (int c = threadIdx.x; c < p.padded; c += 256) h[t * p.padded + c] = used && c < p.d ? to_f32(from[c]) : 0.f;
  }
}

// Eight values of a token, at the columns that load8 gives a lane.
template <bool VEC, int W>
__device__ __forceinline__ void few_values(const float* h, int lane, float2 (&v)[W / 2]) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const float4 a = *reinterpret_cast<const float4*>(h + lane * W + 4 * i);
      v[2 * i] = make_float2(a.x, a.y);
      v[2 * i + 1] = make_float2(a.z, a.w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) v[i] = make_float2(h[64 * i + lane], h[64 * i + 32 + lane]);
  }
}

// 256 columns of four rows of the weight (zeros outside), on their way.
template <typename T, bool VEC>
struct FewRows {
  Pack<T, 8> w[kFewRows];
  __device__ __forceinline__ void fetch(const XentFew& p, long long row0, int c0, int lane) {
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
      const T* row = static_cast<const T*>(p.weight) + (row0 + r) * p.weight_row;
      const int d = row0 + r < p.vocab ? p.d : 0;
      if constexpr (VEC) {
        const int c = c0 + lane * 8;
#pragma unroll
        for (int i = 0; i < int(sizeof(w[r]) / 16); ++i)
          reinterpret_cast<uint4*>(&w[r])[i] = c < d ? reinterpret_cast<const uint4*>(row + c)[i] : make_uint4(0, 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = c0 + j * 32 + lane;
          w[r].v[j] = c < d ? row[c] : from_f32<T>(0.f);
        }
      }
    }
  }
};

// The logits of rows row0 .. row0 + 3: a lane's is that of row lane / N and token lane % N.  (N == 4: of the lanes below 16.)
// `ahead` holds the rows' first columns; then those of the rows from `next` on.
template <typename T, bool VEC, int N>
__device__ __forceinline__ float few_logits(const XentFew& p, const float* h, long long row0, long long next, int lane,
                                            FewRows<T, VEC>& ahead) {
  constexpr int kAll32 = kFewRows * N;
  float2 acc[kFewRows][N];
#pragma unroll
  for (int r = 0; r < kFewRows; ++r)
#pragma unroll
    for (int t = 0; t < N; ++t) acc[r][t] = both(0.f);
  for (int c0 = 0; c0 < p.d; c0 += kChunk) {
    float w[kFewRows][8];
#pragma unroll
    for (int r = 0; r < kFewRows; ++r)
#pragma unroll
      for (int j = 0; j < 8; ++j) w[r][j] = to_f32(ahead.w[r].v[j]);
    const bool last = c0 + kChunk >= p.d;
    ahead.fetch(p, last ? next : row0, last ? 0 : c0 + kChunk, lane);
#pragma unroll
    for (int t = 0; t < N; ++t) {
      float2 v[4];
      few_values<VEC, 8>(h + t * p.padded + c0, lane, v);
#pragma unroll
      for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[r][t] = fma2(make_float2(w[r][2 * i], w[r][2 * i + 1]), v[i], acc[r][t]);
    }
  }
  float v[kAll32];
#pragma unroll
  for (int i = 0; i < kAll32; ++i) v[i] = acc[i / N][i % N].x + acc[i / N][i % N].y;
  // at each step a lane keeps one half of its sums and takes its partner's parts of them
#pragma unroll
  for (int o = kAll32 / 2; o; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float mine = upper ? v[i + o] : v[i], theirs = upper ? v[i] : v[i + o];
      v[i] = mine + __shfl_xor_sync(kAll, theirs, o);
    }
  }
  if constexpr (N == 4) v[0] += __shfl_xor_sync(kAll, v[0], 16);
  return v[0];
}

// Tokens that count.  (a warp)
__device__ __forceinline__ int few_count(const XentFew& p, int lane) {
  return __popc(__ballot_sync(kAll, lane < p.tokens && p.targets[lane] != p.ignore));
}

// Largest logit and sum of exponentials relative to it, of two sets.
__device__ __forceinline__ void few_join(float& top, float& sum, float top2, float sum2) {
  const float m = fmaxf(top, top2), base = m == -INFINITY ? 0.f : m;
  sum = sum * few_exp(top - base) + sum2 * few_exp(top2 - base);
  top = m;
}

// Forward: the statistics of the block's rows for each token, and the targets' logits.  Backward: the logits' gradient.
template <typename T, bool VEC, int N, bool BACKWARD>
__global__ void __launch_bounds__(256, 2) k_few_logits(const XentFew p) {
  extern __shared__ __align__(16) float h[];
  __shared__ float2 each[8][N];
  take_turn();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane % N, r = lane / N;
  const bool mine = r < kFewRows;
  const long long first = ((long long)blockIdx.x * 8 + warp) * kFewRows, step = (long long)gridDim.x * kFewTile;
  FewRows<T, VEC> ahead;
  ahead.fetch(p, first, 0, lane);
  few_hidden<T, N>(p, h);
  const long long target = t < p.tokens && mine ? p.targets[t] : -1;  // (one that is ignored meets no reader)
  float coef = 0.f, lse = 0.f;
  if constexpr (BACKWARD) {
    const int count = few_count(p, lane);
    if (t < p.tokens && p.targets[t] != p.ignore) {
      coef = p.reduction == 0 ? p.grad[t * p.grad_step] : p.reduction == 1 ? p.grad[0] / float(count) : p.grad[0];
      if (p.targets[t] < 0 || p.targets[t] >= p.vocab) coef = __int_as_float(0x7FC00000);
      lse = p.lse_in[t];
    } else {
      lse = INFINITY;  // (no token: whatever a row holds, exp gives 0)
    }
  }
  __syncthreads();
  float top = -INFINITY, sum = 0.f;
  for (long long row0 = first; row0 < p.vocab; row0 += step) {
    const float v = few_logits<T, VEC, N>(p, h, row0, row0 + step, lane, ahead);
    const long long row = row0 + r;
    if (!mine || row >= p.vocab) continue;
    if constexpr (BACKWARD) {
      p.g[row * N + t] = lse == INFINITY && coef == 0.f ? 0.f : coef * (few_exp(v - lse) - (row == target ? 1.f : 0.f));
    } else {
      if (row == target) p.target_logit[t] = v;
      few_join(top, sum, v, 1.f);
    }
  }
  if constexpr (!BACKWARD) {
#pragma unroll
    for (int o = N; o < 32; o *= 2)
      few_join(top, sum, __shfl_xor_sync(kAll, top, o), __shfl_xor_sync(kAll, sum, o));
    if (lane < N) each[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x >= N) return;
    top = each[0][t].x;
    sum = each[0][t].y;
    for (int w = 1; w < 8; ++w) few_join(top, sum, each[w][t].x, each[w][t].y);
    p.part[t * gridDim.x + blockIdx.x] = make_float2(top, sum);
  }
}

// The losses, a warp for each token, and their sum or mean.  The last steps are in 64 bits: lse is several times as large as
// the loss.
__global__ void __launch_bounds__(256) k_few_join(const XentFew p) {
  take_turn();
  __shared__ double each[8];
  const int lane = threadIdx.x & 31, t = threadIdx.x >> 5;
  const int count = few_count(p, lane);
  if (t < p.tokens) {
    const long long target = p.targets[t];
    float top = -INFINITY, sum = 0.f;
    constexpr int kAhead = 5;  // loads on their way
    for (int i = lane; i < p.blocks; i += 32 * kAhead) {
      float2 o[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        o[k] = i + 32 * k < p.blocks ? p.part[t * p.blocks + i + 32 * k] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) few_join(top, sum, o[k].x, o[k].y);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1)
      few_join(top, sum, __shfl_xor_sync(kAll, top, o), __shfl_xor_sync(kAll, sum, o));
    if (lane == 0) {
      const bool used = target != p.ignore;
      const double lse = double(top) + log(double(sum));
      const float loss = !used                                ? 0.f
                         : target < 0 || target >= p.vocab ? __int_as_float(0x7FC00000)
                                                               : float(lse - double(p.target_logit[t]));
      p.lse_out[t] = used ? float(lse) : 0.f;
      if (p.reduction == 0) p.losses[t] = loss;
      each[t] = double(loss);
    }
  }
  __syncthreads();
  if (threadIdx.x || p.reduction == 0) return;
  double sum = 0;
  for (int i = 0; i < p.tokens; ++i) sum += each[i];
  p.losses[0] = float(p.reduction == 1 ? sum / count : sum);
}

// W columns of a lane beside each other (VEC) or 32 apart, W * 32 of a warp from c0 on.
template <typename T, bool VEC, int W>
__device__ __forceinline__ void few_load(const T* row, int c0, int lane, int d, float2 (&v)[W / 2]) {
  if constexpr (VEC) {
    const int c = c0 + lane * W;
    Pack<T, W> a{};
    if (c < d) {
      constexpr int kBytes = int(sizeof(a));
      if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(&a) = *reinterpret_cast<const uint2*>(row + c);
      else
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(&a)[i] = reinterpret_cast<const uint4*>(row + c)[i];
    }
#pragma unroll
    for (int i = 0; i < W / 2; ++i) v[i] = make_float2(to_f32(a.v[2 * i]), to_f32(a.v[2 * i + 1]));
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      const int c = c0 + 64 * i + lane;
      v[i] = make_float2(c < d ? to_f32(row[c]) : 0.f, c + 32 < d ? to_f32(row[c + 32]) : 0.f);
    }
  }
}
template <typename T, bool VEC, int W>
__device__ __forceinline__ void few_store(T* row, int c0, int lane, int d, const float2 (&v)[W / 2]) {
  if constexpr (VEC) {
    const int c = c0 + lane * W;
    if (c >= d) return;
    Pack<T, W> a;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      a.v[2 * i] = from_f32<T>(v[i].x);
      a.v[2 * i + 1] = from_f32<T>(v[i].y);
    }
    constexpr int kBytes = int(sizeof(a));
    if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(row + c) = *reinterpret_cast<const uint2*>(&a);
    else
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(row + c)[i] = reinterpret_cast<const uint4*>(&a)[i];
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      const int c = c0 + 64 * i + lane;
      if (c < d) row[c] = from_f32<T>(v[i].x);
      if (c + 32 < d) row[c + 32] = from_f32<T>(v[i].y);
    }
  }
}

// Both products of the logits' gradient.  A block takes a set of columns (kWide) and its warps four rows of the weight in
// turn; p.ranges blocks share a set.
template <typename T, bool VEC, int N>
__global__ void __launch_bounds__(256, 2) k_few_products(const XentFew p) {
  constexpr int kCols = 32 / N, kWide = 32 * kCols;  // columns of a lane, of a warp
  __shared__ float part[8][32][32];
  take_turn();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int set = int(blockIdx.x) / p.ranges, range = int(blockIdx.x) - set * p.ranges, c0 = set * kWide;
  const auto col = [&](int j) { return VEC ? lane * kCols + j : 32 * j + lane; };
  float2 x[N][kCols / 2], acc[N][kCols / 2];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const bool used = n < p.tokens && p.targets[n] != p.ignore;
    const T* from = static_cast<const T*>(p.hidden) + n * p.hidden_row + c0;
    float v[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) v[j] = used && c0 + col(j) < p.d ? to_f32(from[col(j)]) : 0.f;
#pragma unroll
    for (int j = 0; j < kCols / 2; ++j) {
      x[n][j] = make_float2(v[2 * j], v[2 * j + 1]);
      acc[n][j] = both(0.f);
    }
  }
  for (long long row0 = (range * 8ll + warp) * kFewRows; row0 < p.vocab; row0 += p.ranges * (8ll * kFewRows)) {
    float2 w[kFewRows][kCols / 2];
    float4 f[kFewRows][N / 4];
#pragma unroll
    for (int b = 0; b < kFewRows; ++b) {
      const bool on = row0 + b < p.vocab;
      if (p.sums)
        few_load<T, VEC, kCols>(static_cast<const T*>(p.weight) + (row0 + b) * p.weight_row, c0, lane, on ? p.d : 0, w[b]);
#pragma unroll
      for (int n = 0; n < N / 4; ++n)
        f[b][n] = on ? reinterpret_cast<const float4*>(p.g + (row0 + b) * N)[n] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int b = 0; b < kFewRows; ++b) {
      float2 dw[kCols / 2];
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) dw[j] = both(0.f);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float4 q = f[b][n / 4];
        const float g = n % 4 == 0 ? q.x : n % 4 == 1 ? q.y : n % 4 == 2 ? q.z : q.w;
#pragma unroll
        for (int j = 0; j < kCols / 2; ++j) {
          dw[j] = fma2(both(g), x[n][j], dw[j]);
          if (p.sums) acc[n][j] = fma2(both(g), w[b][j], acc[n][j]);
        }
      }
      if (p.dweight && row0 + b < p.vocab)
        few_store<T, VEC, kCols>(static_cast<T*>(p.dweight) + (row0 + b) * p.d, c0, lane, p.d, dw);
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int j = 0; j < kCols / 2; ++j) {
      part[warp][n * kCols + 2 * j][lane] = acc[n][j].x;
      part[warp][n * kCols + 2 * j + 1][lane] = acc[n][j].y;
    }
  __syncthreads();
  for (int i = warp; i < 32; i += 8) {
    float v = part[0][i][lane];
    for (int k = 1; k < 8; ++k) v += part[k][i][lane];
    const int n = i / kCols, j = i % kCols;
    if (n < p.tokens && c0 + col(j) < p.d) p.sums[((long long)n * p.ranges + range) * p.padded + c0 + col(j)] = v;
  }
}

// The gradient of H from the blocks' sums: 32 columns of a token for each block.
template <typename T>
__global__ void __launch_bounds__(1024) k_few_finish(const XentFew p) {
  take_turn();
  __shared__ float part[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, strips = (p.d + 31) / 32;
  const int t = blockIdx.x / strips, c0 = (blockIdx.x - t * strips) * 32;
  const float* from = p.sums + (long long)t * p.ranges * p.padded + c0 + tx;
  float s = 0.f;
  if (c0 + tx < p.d)
#pragma unroll 4
    for (int i = ty; i < p.ranges; i += 32) s += from[(long long)i * p.padded];
  part[ty][tx] = s;
  __syncthreads();
  const float all = warp_sum(part[tx][ty]);
  if (tx == 0 && c0 + ty < p.d)
    static_cast<T*>(p.dhidden)[(long long)t * p.d + c0 + ty] = from_f32<T>(p.targets[t] != p.ignore ? all : 0.f);
}

template <typename T, bool VEC, int N>
cudaError_t few_launch_n(const XentFew& p, bool backward, cudaStream_t st) {
  // (above 48 KB where it is near, so that a launch raises the kernel's limit: what is not dynamic counts too)
  size_t smem = size_t(N) * p.padded * 4;
  if (smem > 40 * 1024) smem = std::max<size_t>(smem, 48 * 1024 + 16);
  const Shape s{unsigned(p.blocks), 256, smem, 0};
  if (!backward) {
    const cudaError_t e = launch(k_few_logits<T, VEC, N, false>, s, st, p);
    return e != cudaSuccess ? e : launch(k_few_join, Shape{1, 256, 0, 0}, st, p);
  }
  cudaError_t e = launch(k_few_logits<T, VEC, N, true>, s, st, p);
  if (e != cudaSuccess) return e;
  constexpr int kWide = 32 * (32 / N);
  e = launch(k_few_products<T, VEC, N>, Shape{unsigned((p.d + kWide - 1) / kWide * p.ranges), 256, 0, 0}, st, p);
  if (e != cudaSuccess || !p.dhidden) return e;
  return launch(k_few_finish<T>, Shape{unsigned((p.d + 31) / 32 * p.tokens), 1024, 0, 0}, st, p);
}

template <typename T>
cudaError_t few_launch(const XentFew& p, bool vec, bool backward, cudaStream_t st) {
  if (p.tokens <= 4) return vec ? few_launch_n<T, true, 4>(p, backward, st) : few_launch_n<T, false, 4>(p, backward, st);
  return vec ? few_launch_n<T, true, 8>(p, backward, st) : few_launch_n<T, false, 8>(p, backward, st);
}

}  // namespace
}  // namespace efcp
