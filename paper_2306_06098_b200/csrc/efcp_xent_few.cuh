// Linear cross entropy of up to eight tokens (the formulas stand in include/efcp.h): the layer's weight is what there is to
// read, and its gradient to write; tiles of the tensor cores would be empty but for a few rows.
//
// The hidden states lie in shared memory in fp32.  A warp takes four rows of the weight, multiplies them with all
// tokens in fp32 (two products to an instruction), and adds up its lanes' parts so that each lane ends up with one logit.
// Backward a block does that for 32 rows, turns the logits into their gradient in shared memory, and then its warps, on
// columns of their own, read the rows once more out of the cache: they hold the gradient of the hidden states in registers
// and write the gradient of the weight.  The blocks' sums are added up in order.
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

// 8 (or fewer) values of a token, at the columns that load8 gives a lane
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

// The logits of rows row0 .. row0 + 3: a lane's is that of row lane / N and token lane % N.  (N == 4: of the lanes below 16.)
template <typename T, bool VEC, int N>
__device__ __forceinline__ float few_logits(const XentFew& p, const float* h, long long row0, int lane) {
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
      load8<T, VEC>(static_cast<const T*>(p.weight) + (row0 + r) * p.weight_row, c0, lane, row0 + r < p.vocab ? p.d : 0,
                    w[r]);
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

// Largest logit and sum of exponentials relative to it, of two sets.
__device__ __forceinline__ void few_join(float& top, float& sum, float top2, float sum2) {
  const float m = fmaxf(top, top2), base = m == -INFINITY ? 0.f : m;
  sum = sum * few_exp(top - base) + sum2 * few_exp(top2 - base);
  top = m;
}

template <typename T, bool VEC, int N>
__global__ void __launch_bounds__(256, 2) k_few_forward(const XentFew p) {
  extern __shared__ __align__(16) float h[];
  __shared__ float2 each[8][N];
  take_turn();
  few_hidden<T, N>(p, h);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane % N, r = lane / N;
  const bool mine = r < kFewRows;
  const long long target = t < p.tokens && mine ? p.targets[t] : -1;  // (one that is ignored meets no reader)
  float top = -INFINITY, sum = 0.f;
  for (long long row0 = ((long long)blockIdx.x * 8 + warp) * kFewRows; row0 < p.vocab;
       row0 += (long long)gridDim.x * kFewTile) {
    const float v = few_logits<T, VEC, N>(p, h, row0, lane);
    const long long row = row0 + r;
    if (!mine || row >= p.vocab) continue;
    if (row == target) p.target_logit[t] = v;
    few_join(top, sum, v, 1.f);
  }
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

// The losses, a warp for each token, and their sum or mean.  The last steps are in 64 bits: lse is several times as large as
// the loss.
__global__ void __launch_bounds__(256) k_few_join(const XentFew p) {
  take_turn();
  __shared__ double each[8];
  const int lane = threadIdx.x & 31, t = threadIdx.x >> 5;
  int count = 0;
  for (int i = 0; i < p.tokens; ++i) count += p.targets[i] != p.ignore;
  if (t < p.tokens) {
    const long long target = p.targets[t];
    float top = -INFINITY, sum = 0.f;
    for (int i = lane; i < p.blocks; i += 32) {
      const float2 o = p.part[t * p.blocks + i];
      few_join(top, sum, o.x, o.y);
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

// K: sets of columns of a warp
template <typename T, bool VEC, int N, int K>
__global__ void __launch_bounds__(256, 2) k_few_backward(const XentFew p) {
  constexpr int kCols = 32 / N, kWide = 32 * kCols;  // columns of a lane, of a warp
  extern __shared__ __align__(16) float h[];
  __shared__ __align__(16) float g[2][kFewTile][N];
  take_turn();
  few_hidden<T, N>(p, h);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane % N, r = lane / N;
  // the factor on the token's gradient
  float coef = 0.f, lse = 0.f;
  long long target = -1;
  {
    int count = 0;
    for (int i = 0; i < p.tokens; ++i) count += p.targets[i] != p.ignore;
    if (t < p.tokens && p.targets[t] != p.ignore) {
      target = p.targets[t];
      coef = p.reduction == 0 ? p.grad[t * p.grad_step] : p.reduction == 1 ? p.grad[0] / float(count) : p.grad[0];
      if (target < 0 || target >= p.vocab) coef = __int_as_float(0x7FC00000);
      lse = p.lse_in[t];
    }
  }
  // sets of columns: several for each warp, or rows shared out to the warps of one
  const int sets = (p.d + kWide - 1) / kWide, shares = sets >= 8 ? 1 : 8 / sets;
  const int set = sets >= 8 ? warp : warp % sets, share = sets >= 8 ? 0 : warp / sets;
  float2 acc[K][N][kCols / 2];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) acc[k][i][j] = both(0.f);
  int turn = 0;
  for (long long tile = (long long)blockIdx.x * kFewTile; tile < p.vocab; tile += (long long)gridDim.x * kFewTile, turn ^= 1) {
    const long long row = tile + warp * kFewRows + r;
    const float v = few_logits<T, VEC, N>(p, h, tile + warp * kFewRows, lane);
    if (r < kFewRows)
      g[turn][warp * kFewRows + r][t] =
          row < p.vocab && t < p.tokens ? coef * (few_exp(v - lse) - (row == target ? 1.f : 0.f)) : 0.f;
    __syncthreads();  // (the other half of g is free by the time that it is written again)
    if (share >= shares) continue;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = (set + 8 * k) * kWide;
      if (c0 >= p.d) continue;
      for (int i = share; i < kFewTile && tile + i < p.vocab; i += 2 * shares) {
        // two rows at a time, for one read of the hidden states
        float2 w[2][kCols / 2], dw[2][kCols / 2];
        float f[2][N];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int at = i + b * shares;
          const bool on = at < kFewTile && tile + at < p.vocab;
#pragma unroll
          for (int j = 0; j < kCols / 2; ++j) dw[b][j] = w[b][j] = both(0.f);
          if (on && p.sums)
            few_load<T, VEC, kCols>(static_cast<const T*>(p.weight) + (tile + at) * p.weight_row, c0, lane, p.d, w[b]);
#pragma unroll
          for (int n = 0; n < N; n += 4)
            *reinterpret_cast<float4*>(&f[b][n]) =
                on ? *reinterpret_cast<const float4*>(&g[turn][at][n]) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
          float2 x[kCols / 2];
          few_values<VEC, kCols>(h + n * p.padded + c0, lane, x);
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) {
              dw[b][j] = fma2(both(f[b][n]), x[j], dw[b][j]);
              acc[k][n][j] = fma2(both(f[b][n]), w[b][j], acc[k][n][j]);
            }
        }
        if (p.dweight) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int at = i + b * shares;
            if (at < kFewTile && tile + at < p.vocab)
              few_store<T, VEC, kCols>(static_cast<T*>(p.dweight) + (tile + at) * p.d, c0, lane, p.d, dw[b]);
          }
        }
      }
    }
  }
  if (!p.sums) return;
  // the shares of a set are added up in order, in the place of the hidden states
  for (int s = 1; s < shares; ++s) {
    __syncthreads();
    const int c0 = set * kWide;
    if (share == s)
#pragma unroll
      for (int n = 0; n < N; ++n) few_store<float, VEC, kCols>(h + n * p.padded, c0, lane, p.padded, acc[0][n]);
    __syncthreads();
    if (share == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float2 x[kCols / 2];
        few_values<VEC, kCols>(h + n * p.padded + c0, lane, x);
#pragma unroll
        for (int j = 0; j < kCols / 2; ++j) acc[0][n][j] = add2(acc[0][n][j], x[j]);
      }
  }
  if (share) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c0 = (set + 8 * k) * kWide;
    if (c0 >= p.d) continue;
#pragma unroll
    for (int n = 0; n < N; ++n)
      few_store<float, VEC, kCols>(p.sums + ((long long)n * gridDim.x + blockIdx.x) * p.padded, c0, lane, p.padded, acc[k][n]);
  }
}

// The gradient of H from the blocks' sums: 32 columns of a token for each block.
template <typename T>
__global__ void __launch_bounds__(1024) k_few_finish(const XentFew p) {
  take_turn();
  __shared__ float part[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, strips = (p.d + 31) / 32;
  const int t = blockIdx.x / strips, c0 = (blockIdx.x - t * strips) * 32;
  const float* from = p.sums + (long long)t * p.blocks * p.padded + c0 + tx;
  float s = 0.f;
#pragma unroll 8
  for (int i = ty; i < p.blocks; i += 32) s += from[(long long)i * p.padded];
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
    const cudaError_t e = launch(k_few_forward<T, VEC, N>, s, st, p);
    return e != cudaSuccess ? e : launch(k_few_join, Shape{1, 256, 0, 0}, st, p);
  }
  const cudaError_t e = p.d <= 256 * (32 / N) ? launch(k_few_backward<T, VEC, N, 1>, s, st, p)
                                              : launch(k_few_backward<T, VEC, N, 2>, s, st, p);
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
