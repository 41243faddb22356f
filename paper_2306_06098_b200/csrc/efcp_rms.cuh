// Root-mean-square norm of a residual stream, forward, backward and with an output in 8 bits, and dropout of
// rows (the formulas stand in include/efcp.h).
//
// Every input is read once, every output written once.  The plain kernels here, for what is little and for rows that are long, wait
// on latency more than on the memory (1531 x 1111 fp32 backward: 21 % of its rate, 36 % of the issue slots).  A row is shared out over one
// to 32 warps whose lanes keep it in registers between the sum and the result (K chunks a warp); rows longer than
// that (K == 0) are walked twice, the second time out of the cache.  Backward a thread keeps its columns
// over all rows that its block takes, so the weight's gradient grows in registers; the blocks' sums are
// added up in a fixed order by a second kernel.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_rms.h"
#include "efcp_rms_ring.cuh"
#include "efcp_rows.cuh"

namespace efcp {
namespace {

constexpr int kMaxRowWarps = 32;

// Sum (or maximum) over the warps of a row; `slot` tells the exchanges of one row apart, and a barrier lies between
// two uses of the same slot.
template <bool MAX>
__device__ __forceinline__ float row_join(float v, int warps, int group, int w, int slot) {
  __shared__ float part[4][kMaxRowWarps];
  if constexpr (MAX) v = lanes_max(v, 32);
  else v = warp_sum(v);
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) part[slot][group * warps + w] = v;
  __syncthreads();
  float all = part[slot][group * warps];
  for (int i = 1; i < warps; ++i) {
    const float o = part[slot][group * warps + i];
    if constexpr (MAX) all = larger(all, o);
    else all += o;
  }
  return all;
}

template <typename T, bool VEC>
struct Row {
  const Rms& p;
  long long row;
  int lane;
  DropKey key;
  // h in fp32, rounded to its type; stored where it is an output
  __device__ __forceinline__ void sum8(int c0, bool on, float (&v)[8]) const {
    load8<T, VEC>(static_cast<const T*>(p.x) + row * p.x_row, c0, lane, p.d, v);
    float r[8];
    if (p.residual)
      load8<T, VEC>(static_cast<const T*>(p.residual) + row * p.residual_row, c0, lane, p.d, r);
    if (p.drop.threshold)
      drop8<VEC>(v, (unsigned long long)row * p.d + c0, lane, key, p.drop);
    if (p.residual) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    if (p.h) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rounded<T>(v[j]);
      if (on) store8<T, VEC>(static_cast<T*>(p.h) + row * p.d, c0, lane, p.d, v);
    }
  }
  // the same once more, from where it lies
  __device__ __forceinline__ void again8(int c0, float (&v)[8]) const {
    if (p.h) load8<T, VEC>(static_cast<const T*>(p.h) + row * p.d, c0, lane, p.d, v);
    else load8<T, VEC>(static_cast<const T*>(p.x) + row * p.x_row, c0, lane, p.d, v);
  }
  __device__ __forceinline__ void norm8(int c0, float rstd, float (&v)[8]) const {
    float w[8];
    if (p.weight) load8_param<VEC>(p.weight, p.param_dtype, c0, lane, p.d, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p.weight ? v[j] * rstd * w[j] : v[j] * rstd;
  }
};

__device__ __forceinline__ float max8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = larger(m, fabsf(v[j]));
  return m;
}

template <bool VEC, bool E4M3>
__device__ __forceinline__ void store_q8(unsigned char* row, int c0, int lane, int d,
                                         const float (&v)[8], const float (&s)[8]) {
  if constexpr (VEC) {
    const int col = c0 + lane * 8;
    if (col < d) {
      uint2 q = {0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q.x |= quantized<E4M3>(v[j], s[j], inverse_of(s[j])) << (8 * j);
        q.y |= quantized<E4M3>(v[4 + j], s[4 + j], inverse_of(s[4 + j])) << (8 * j);
      }
      *reinterpret_cast<uint2*>(row + col) = q;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = c0 + j * 32 + lane;
      if (col < d) row[col] = (unsigned char)quantized<E4M3>(v[j], s[j], inverse_of(s[j]));
    }
  }
}

// The scales of a lane's elements in a chunk of blocks of 32, 64 or 128 columns, written by one lane a block.
template <bool VEC>
__device__ __forceinline__ void block_scales(const Rms& p, float* scales, int c0, int lane,
                                             const float (&v)[8], float (&s)[8]) {
  if constexpr (VEC) {
    const int lanes = p.block / 8, col = c0 + lane * 8;
    const float one = scale_of(lanes_max(max8(v), lanes), p.most);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = one;
    if (lane % lanes == 0 && col < p.d) scales[col >> p.block_shift] = one;
  } else {
    const int strips = p.block / 32;
    float top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = lanes_max(fabsf(v[j]), 32);
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
      if (o < strips) {
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = larger(top[j], top[j ^ o]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top[j] = t[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = scale_of(top[j], p.most);
      const int col = c0 + j * 32;
      if (lane == 0 && j % strips == 0 && col < p.d) scales[col >> p.block_shift] = s[j];
    }
  }
}

// QUANT 0: y in T; 1: e4m3; 2: int8
template <typename T, bool VEC, int K, int QUANT>
__global__ void __launch_bounds__(K == 0 ? 1024 : 512, K == 0 ? 1 : 2) k_rms_forward(const Rms p) {
  take_turn();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / p.warps, w = warp - group * p.warps;
  const long long row = (long long)blockIdx.x * p.groups + group;
  const bool on = row < p.rows;
  Row<T, VEC> r{p, on ? row : p.rows - 1, lane, drop_key(p.drop)};  // (idle warps meet the barriers)
  const int step = p.warps * kChunk;
  constexpr int kKept = K ? K : 1;
  float v[kKept][8];
  float sum = 0.f;
  const auto add = [&](const float(&a)[8]) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += a[j] * a[j];
    sum += s * p.inv_d;  // (the mean, not the sum, has to stay in range)
  };
  if constexpr (K > 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = w * kChunk + k * step;
      if (c0 < p.d) {
        r.sum8(c0, on, v[k]);
        add(v[k]);
      }
    }
  } else {
    for (int c0 = w * kChunk; c0 < p.d; c0 += step) {
      r.sum8(c0, on, v[0]);
      add(v[0]);
    }
  }
  const float rstd = rsqrtf(row_join<false>(sum, p.warps, group, w, 0) + p.eps);
  if (on && w == 0 && lane == 0 && p.rstd) p.rstd[row] = rstd;
  const auto chunks = [&](auto f) {  // f(chunk's first column, z of the lane)
    if constexpr (K > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c0 = w * kChunk + k * step;
        if (c0 < p.d) f(c0, v[k]);
      }
    } else {
      for (int c0 = w * kChunk; c0 < p.d; c0 += step) {
        r.again8(c0, v[0]);
        r.norm8(c0, rstd, v[0]);
        f(c0, v[0]);
      }
    }
  };
  if constexpr (K > 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = w * kChunk + k * step;
      if (c0 < p.d) r.norm8(c0, rstd, v[k]);
    }
  }
  if constexpr (QUANT == 0) {
    chunks([&](int c0, const float(&z)[8]) {
      if (on) store8<T, VEC>(static_cast<T*>(p.y) + row * p.d, c0, lane, p.d, z);
    });
  } else {
    unsigned char* q = static_cast<unsigned char*>(p.y) + r.row * p.d;
    float* scales = p.scales + r.row * p.blocks;
    float s[8];
    if (p.block == 0) {
      float top = 0.f;
      chunks([&](int, const float(&z)[8]) { top = larger(top, max8(z)); });
      const float one = scale_of(row_join<true>(top, p.warps, group, w, 1), p.most);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = one;
      if (on && w == 0 && lane == 0) scales[0] = one;
    }
    chunks([&](int c0, const float(&z)[8]) {
      if (!on) return;  // (whole warps)
      if (p.block) block_scales<VEC>(p, scales, c0, lane, z, s);
      store_q8<VEC, QUANT == 1>(q, c0, lane, p.d, z, s);
    });
  }
}

// p.x is h; a group of warps takes the rows slot, slot + slots, ...
template <typename T, bool VEC, int K>
__global__ void __launch_bounds__(K == 0 ? 1024 : 512) k_rms_backward(const Rms p) {
  take_turn();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / p.warps, w = warp - group * p.warps;
  const long long slots = (long long)gridDim.x * p.groups;
  const long long slot = (long long)blockIdx.x * p.groups + group;
  const int step = p.warps * kChunk;
  const DropKey key = drop_key(p.drop);
  constexpr int kKept = K ? K : 1;
  float dy[kKept][8], h[kKept][8], dw[kKept][8], wt[8];
#pragma unroll
  for (int k = 0; k < kKept; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[k][j] = 0.f;
  const long long turns = (p.rows + slots - 1) / slots;
  for (long long i = 0; i < turns; ++i) {
    const bool on = slot + i * slots < p.rows;
    const long long row = on ? slot + i * slots : p.rows - 1;
    const float r = p.rstd[row];
    const auto load = [&](int c0, float(&a)[8], float(&b)[8]) {
      load8<T, VEC>(static_cast<const T*>(p.dy) + row * p.dy_row, c0, lane, p.d, a);
      load8<T, VEC>(static_cast<const T*>(p.x) + row * p.x_row, c0, lane, p.d, b);
    };
    const auto weight = [&](int c0) {
      if (p.weight) load8_param<VEC>(p.weight, p.param_dtype, c0, lane, p.d, wt);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) wt[j] = 1.f;
    };
    float sum = 0.f;
    const auto add = [&](int c0, const float(&a)[8], const float(&b)[8]) {
      weight(c0);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s += a[j] * wt[j] * b[j];
      sum += s;
    };
    if constexpr (K > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c0 = w * kChunk + k * step;
        if (c0 < p.d) load(c0, dy[k], h[k]);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c0 = w * kChunk + k * step;
        if (c0 < p.d) add(c0, dy[k], h[k]);
      }
    } else {
      for (int c0 = w * kChunk; c0 < p.d; c0 += step) {
        load(c0, dy[0], h[0]);
        add(c0, dy[0], h[0]);
      }
    }
    const float c = row_join<false>(sum, p.warps, group, w, int(i & 1)) * p.inv_d * r * r;
    const auto finish = [&](int c0, const float(&a)[8], const float(&b)[8], float(&acc)[8]) {
      if (!on) return;
      float dz[8];
      if (p.dh) load8<T, VEC>(static_cast<const T*>(p.dh) + row * p.dh_row, c0, lane, p.d, dz);
      weight(c0);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = r * (a[j] * wt[j] - b[j] * c);
        dz[j] = p.dh ? g + dz[j] : g;
        acc[j] += a[j] * b[j] * r;
      }
      if (p.dresidual)
        store8<T, VEC>(static_cast<T*>(p.dresidual) + row * p.d, c0, lane, p.d, dz);
      if (p.dx) {
        if (p.drop.threshold)
          drop8<VEC>(dz, (unsigned long long)row * p.d + c0, lane, key, p.drop);
        store8<T, VEC>(static_cast<T*>(p.dx) + row * p.d, c0, lane, p.d, dz);
      }
    };
    if constexpr (K > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c0 = w * kChunk + k * step;
        if (c0 < p.d) finish(c0, dy[k], h[k], dw[k]);
      }
    } else {
      for (int c0 = w * kChunk; c0 < p.d; c0 += step) {
        load(c0, dy[0], h[0]);
        finish(c0, dy[0], h[0], dw[0]);
      }
    }
  }
  if (K > 0 && p.part) {
#pragma unroll
    for (int k = 0; k < kKept; ++k) {
      const int c0 = w * kChunk + k * step;
      if (c0 < p.d) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int col = col_of<VEC>(c0, lane, j);
          if (col < p.d) p.part[slot * p.d + col] = dw[k][j];
        }
      }
    }
  }
}

// Partial sums of the weight's gradient for rows too long for registers: a warp takes 256 columns of every
// `slots`-th row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_rms_dweight(const Rms p) {
  take_turn();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned tiles = unsigned(p.d + kChunk - 1) / kChunk, y = blockIdx.x / tiles;
  const int c0 = int(blockIdx.x - y * tiles) * kChunk;
  const long long slot = (long long)y * 8 + warp, slots = (long long)(gridDim.x / tiles) * 8;
  float acc[8] = {};
  for (long long row = slot; row < p.rows; row += slots) {
    float a[8], b[8];
    load8<T, VEC>(static_cast<const T*>(p.dy) + row * p.dy_row, c0, lane, p.d, a);
    load8<T, VEC>(static_cast<const T*>(p.x) + row * p.x_row, c0, lane, p.d, b);
    const float r = p.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += a[j] * b[j] * r;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int col = col_of<VEC>(c0, lane, j);
    if (col < p.d) p.part[slot * p.d + col] = acc[j];
  }
}

// dweight from `count` partial sums a column: 32 columns a block, 32 rows of threads.
__global__ void __launch_bounds__(1024) k_rms_dweight_join(const float* part, long long count, int d,
                                                           void* dweight, int param_dtype) {
  take_turn();
  __shared__ float sum[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, col = int(blockIdx.x) * 32 + tx;
  float s = 0.f;
  if (col < d)
#pragma unroll 8
    for (long long i = ty; i < count; i += 32) s += part[i * d + col];
  sum[ty][tx] = s;
  __syncthreads();
  const float all = warp_sum(sum[tx][ty]);
  const int out = int(blockIdx.x) * 32 + ty;
  if (tx == 0 && out < d) store_from_f32(dweight, param_dtype, out, all);
}

// y = dropout(x) (+ residual); a warp takes chunks of rows in turn.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_dropout(const Rms p) {
  take_turn();
  const int lane = threadIdx.x & 31;
  const long long chunks = (p.d + kChunk - 1) / kChunk, all = p.rows * chunks;
  const DropKey key = drop_key(p.drop);
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < all; i += (long long)gridDim.x * 8) {
    const long long row = i / chunks;
    const int c0 = int(i - row * chunks) * kChunk;
    float v[8], r[8];
    load8<T, VEC>(static_cast<const T*>(p.x) + row * p.x_row, c0, lane, p.d, v);
    if (p.residual)
      load8<T, VEC>(static_cast<const T*>(p.residual) + row * p.residual_row, c0, lane, p.d, r);
    if (p.drop.threshold)
      drop8<VEC>(v, (unsigned long long)row * p.d + c0, lane, key, p.drop);
    if (p.residual) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    store8<T, VEC>(static_cast<T*>(p.y) + row * p.d, c0, lane, p.d, v);
  }
}

// The same of rows that lie one behind the other: one row of eights, two to a thread at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout_flat(const Rms p) {
  take_turn();
  const T* const x = static_cast<const T*>(p.x);
  const T* const residual = static_cast<const T*>(p.residual);
  T* const y = static_cast<T*>(p.y);
  const DropKey key = drop_key(p.drop);
  const long long n = p.rows * p.d, eights = n / 8, step = (long long)gridDim.x * 256;
  const auto one = [&](long long g, Eight<T>& a, const Eight<T>& b) {
    float2 v[4], r[4];
    a.get(v);
    if (p.drop.threshold) drop_pairs(v, (unsigned long long)g, key, p.drop);
    if (residual) {
      b.get(r);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = add2(v[i], r[i]);
    }
    a.set(v);
    a.store(y + g * 8);
  };
  for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; g < eights; g += 2 * step) {
    const long long h = g + step;
    const bool both_ = h < eights;
    Eight<T> a[2], b[2];
    a[0].load(x + g * 8);
    if (residual) b[0].load(residual + g * 8);
    if (both_) {
      a[1].load(x + h * 8);
      if (residual) b[1].load(residual + h * 8);
    }
    one(g, a[0], b[0]);
    if (both_) one(h, a[1], b[1]);
  }
  if (blockIdx.x == 0 && threadIdx.x < n - eights * 8) {
    const long long e = eights * 8 + threadIdx.x;
    float v = to_f32(x[e]);
    if (p.drop.threshold)
      v = (drop_keep8((unsigned long long)eights, key, p.drop.threshold) >> threadIdx.x) & 1u ? v * p.drop.scale : 0.f;
    if (residual) v += to_f32(residual[e]);
    y[e] = from_f32<T>(v);
  }
}

inline cudaError_t rms_join(const Rms& p, const RmsLaunch& l) {
  return launch(k_rms_dweight_join, Shape{unsigned((p.d + 31) / 32), 1024, 0, 0}, l.st,
                static_cast<const float*>(p.part), l.parts, p.d, p.dweight, p.param_dtype);
}

template <typename T, bool VEC, int K>
cudaError_t rms_launch_k(const Rms& p, const RmsLaunch& l) {
  const Shape s{l.blocks, unsigned(p.groups * p.warps * 32), 0, 0};
  if (l.op == kRmsBackward) return launch(k_rms_backward<T, VEC, K>, s, l.st, p);
  if (l.op == kRmsE4M3) return launch(k_rms_forward<T, VEC, K, 1>, s, l.st, p);
  if (l.op == kRmsInt8) return launch(k_rms_forward<T, VEC, K, 2>, s, l.st, p);
  return launch(k_rms_forward<T, VEC, K, 0>, s, l.st, p);
}

template <typename T, bool VEC>
cudaError_t rms_launch_vec(const Rms& p, const RmsLaunch& l) {
  if (l.op == kDropout)
    return l.flat ? launch(k_dropout_flat<T>, Shape{l.blocks, 256, 0, 0}, l.st, p)
                  : launch(k_dropout<T, VEC>, Shape{l.blocks, 256, 0, 0}, l.st, p);
  cudaError_t e = l.kept == 1   ? rms_launch_k<T, VEC, 1>(p, l)
                  : l.kept == 2 ? rms_launch_k<T, VEC, 2>(p, l)
                  : l.kept == 4 ? rms_launch_k<T, VEC, 4>(p, l)
                                : rms_launch_k<T, VEC, 0>(p, l);
  if (e != cudaSuccess || l.op != kRmsBackward || !p.part) return e;
  if (l.kept == 0) {
    const unsigned tiles = unsigned(p.d + kChunk - 1) / kChunk;
    e = launch(k_rms_dweight<T, VEC>, Shape{tiles * unsigned(l.parts / 8), 256, 0, 0}, l.st, p);
    if (e != cudaSuccess) return e;
  }
  return rms_join(p, l);
}

template <typename T>
cudaError_t rms_launch(const Rms& p, const RmsLaunch& l) {
  if (l.ringed) {
    const cudaError_t e = l.vec ? rms_launch_ring<T, false>(p, l) : rms_launch_ring<T, true>(p, l);
    if (e != cudaSuccess || !p.part) return e;
    return rms_join(p, l);
  }
  return l.vec ? rms_launch_vec<T, true>(p, l) : rms_launch_vec<T, false>(p, l);
}

}  // namespace
}  // namespace efcp
