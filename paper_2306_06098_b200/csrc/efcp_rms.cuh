// Root-mean-square norm of a residual stream, forward, backward and with an output in 8 bits, and dropout of
// rows (the formulas stand in include/efcp.h).
//
// Memory bounds them: every input is read once, every output written once.  A row is shared out over one
// to 32 warps whose lanes keep it in registers between the sum and the result (K chunks a warp); rows longer than
// that (K == 0) are walked twice, the second time out of the cache.  Backward a thread keeps its columns
// over all rows that its block takes, so the weight's gradient grows in registers; the blocks' sums are
// added up in a fixed order by a second kernel.
#pragma once

#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_rms.h"
#include "efcp_rows.cuh"
#include "efcp_tc.cuh"

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

// The scale of a block whose largest magnitude is `top`: 1 for zeros, NaN where a value is not finite.
__device__ __forceinline__ float scale_of(float top, float most) {
  if (!(top < __int_as_float(0x7F800000))) return __int_as_float(0x7FC00000);
  const float s = top / most;
  return s > 0.f ? s : 1.f;
}

// 1 / s, and 0 for a scale of NaN
__device__ __forceinline__ float inverse_of(float s) { return s == s ? 1.f / s : 0.f; }

// z / s as 8 bits, given 1 / s: the quotient is off by up to two roundings of fp32, so a value that close to the
// border between two 8-bit ones may go either way; 0 in a block whose scale is NaN.
template <bool E4M3>
__device__ __forceinline__ unsigned quantized(float z, float inv) {
  const float q = inv > 0.f ? z * inv : 0.f;
  if constexpr (E4M3) return __nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
  else return unsigned(max(-127, min(127, __float2int_rn(q)))) & 0xFFu;
}
template <bool E4M3>
__device__ __forceinline__ unsigned quantized2(float2 z, float inv) {
  if constexpr (E4M3) {
    const float2 q = inv > 0.f ? make_float2(z.x * inv, z.y * inv) : make_float2(0.f, 0.f);
    return __nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, __NV_E4M3);
  } else {
    return quantized<false>(z.x, inv) | quantized<false>(z.y, inv) << 8;
  }
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
        q.x |= quantized<E4M3>(v[j], inverse_of(s[j])) << (8 * j);
        q.y |= quantized<E4M3>(v[4 + j], inverse_of(s[4 + j])) << (8 * j);
      }
      *reinterpret_cast<uint2*>(row + col) = q;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = c0 + j * 32 + lane;
      if (col < d) row[col] = (unsigned char)quantized<E4M3>(v[j], inverse_of(s[j]));
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
    if (lane % lanes == 0 && col < p.d) scales[col / p.block] = one;
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
      if (lane == 0 && j % strips == 0 && col < p.d) scales[col / p.block] = s[j];
    }
  }
}

// QUANT 0: y in T; 1: e4m3; 2: int8
template <typename T, bool VEC, int K, int QUANT>
__global__ void __launch_bounds__(K == 0 ? 1024 : 512) k_rms_forward(const Rms p) {
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

// ------------------------------------------------------------------ rows through shared memory
// Bulk copies bring whole rows into shared memory while earlier ones are worked on, so that enough bytes are on
// their way without a register being held for them.  Two blocks of eight warps share an SM.  A group of warps
// asks for the next unit of a place when a barrier has told that all of them are done with the one there.

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}

struct RingInput {
  const void* data;
  long long row;  // bytes between rows
};

// A group's view of its ring.
template <int INPUTS>
struct Ring {
  const Rms& p;
  const RmsRing& q;
  unsigned char* data;  // of this group
  uint32_t bars;
  int* gave_up;
  long long first, step, units;  // units of the group: first, first + step, ...
  int group, warp, lane;
  RingInput in[INPUTS];

  __device__ __forceinline__ unsigned char* place(int s, int i) const {
    return data + (s * q.inputs + i) * q.unit_bytes;
  }
  // the warps of the group meet
  __device__ __forceinline__ void meet() const {
    if (p.warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(p.warps * 32) : "memory");
  }
  // (one thread) the group's unit number n into its place
  __device__ __forceinline__ void ask(long long n) const {
    const long long u = first + n * step;
    if (u >= units) return;
    const int s = int(n % q.stages);
    const long long row = u * q.rows;
    const int rows = int(min((long long)q.rows, p.rows - row));
    const uint32_t bar = bars + 8 * s;
    tc::bar_expect(bar, uint32_t(rows * q.row_bytes * q.inputs));
#pragma unroll
    for (int i = 0; i < INPUTS; ++i) {
      if (i >= q.inputs) break;
      const char* from = static_cast<const char*>(in[i].data) + row * in[i].row;
      const uint32_t to = tc::smem_of(place(s, i));
      if (in[i].row == q.row_bytes) bulk_copy(to, from, uint32_t(rows * q.row_bytes), bar);
      else
        for (int r = 0; r < rows; ++r) bulk_copy(to + r * q.row_bytes, from + r * in[i].row, uint32_t(q.row_bytes), bar);
    }
  }
  // Unit number n has arrived.  When the limit passes the work goes on with whatever lies there (the warps of a
  // group keep meeting), no further wait is long, and the status tells.
  __device__ __forceinline__ void await(long long n) const {
    (void)tc::bar_wait(bars + 8 * int(n % q.stages), uint32_t(n / q.stages) & 1, gave_up);
  }
  // Nothing may land in shared memory that the block has left.
  __device__ __forceinline__ void end(long long asked) const {
    if (!*(volatile int*)gave_up) return;
    for (long long n = asked < q.stages ? 0 : asked - q.stages; n < asked; ++n)
      if (first + n * step < units)
        (void)tc::bar_wait(bars + 8 * int(n % q.stages), uint32_t(n / q.stages) & 1, gave_up, tc::kDrainNs);
  }
};

// Barriers, the weight in fp32, and the group that a warp belongs to.  (Up to 8 groups of up to 4 places.)
template <int INPUTS>
__device__ __forceinline__ Ring<INPUTS> ring_begin(const Rms& p, const RmsRing& q, unsigned char* smem,
                                                   int* gave_up) {
  const int warp = threadIdx.x >> 5;
  const uint32_t bars = tc::smem_of(smem);
  if (threadIdx.x == 0) {
    *gave_up = 0;
    for (int i = 0; i < p.groups * q.stages; ++i) tc::bar_init(bars + 8 * i, 1);
    tc::bar_init_fence();
  }
  take_turn();
  float* weight = reinterpret_cast<float*>(smem + q.weight_at);
  if (p.weight)
    for (int c = threadIdx.x; c < p.d; c += blockDim.x) weight[c] = load_as_f32(p.weight, p.param_dtype, c);
  __syncthreads();
  const int g = warp / p.warps;
  return Ring<INPUTS>{p, q, smem + q.data_at + (size_t)g * q.stages * q.inputs * q.unit_bytes,
                      bars + 8 * g * q.stages, gave_up,
                      (long long)blockIdx.x * p.groups + g, (long long)gridDim.x * p.groups,
                      (p.rows + q.rows - 1) / q.rows, g, warp - g * p.warps, int(threadIdx.x) & 31, {}};
}

// Eight elements as they lie in memory.
template <typename T>
struct Eight {
  uint4 raw[sizeof(T) / 2];

  __device__ __forceinline__ void load_shared(uint32_t at) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w)
                   : "r"(at + 16 * i)
                   : "memory");
  }
  __device__ __forceinline__ void store_shared(uint32_t at) const {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16 * i), "r"(raw[i].x),
                   "r"(raw[i].y), "r"(raw[i].z), "r"(raw[i].w)
                   : "memory");
  }
  __device__ __forceinline__ void store(T* to) const {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(to)[i] = raw[i];
  }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        v[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
      } else {
        v[i] = __half22float2(reinterpret_cast<const __half2*>(w)[i]);
      }
    }
  }
  __device__ __forceinline__ void set(const float2 (&v)[4]) {
    uint32_t* w = reinterpret_cast<uint32_t*>(raw);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        w[2 * i] = __float_as_uint(v[i].x);
        w[2 * i + 1] = __float_as_uint(v[i].y);
      } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        reinterpret_cast<__nv_bfloat162*>(w)[i] = __float22bfloat162_rn(v[i]);
      } else {
        reinterpret_cast<__half2*>(w)[i] = __float22half2_rn(v[i]);
      }
    }
  }
};

__device__ __forceinline__ void drop_pairs(float2 (&v)[4], unsigned long long group, const DropKey& key,
                                           const Drop& drop) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { w[2 * i] = v[i].x; w[2 * i + 1] = v[i].y; }
  drop_group(w, group, key, drop.threshold, drop.scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float2(w[2 * i], w[2 * i + 1]);
}

// Sum (or maximum) over the lanes and warps that share a row; `slot` as in row_join.
template <bool MAX, int INPUTS>
__device__ __forceinline__ float ring_join(const Ring<INPUTS>& r, float v, int slot) {
  __shared__ float part[4][8];
  for (int o = r.q.lanes / 2; o; o >>= 1) {
    const float other = __shfl_xor_sync(kAll, v, o);
    if constexpr (MAX) v = larger(v, other);
    else v += other;
  }
  if (r.p.warps == 1) {
    __syncwarp();
    return v;
  }
  float* mine = part[slot] + r.group * r.p.warps;
  if (r.lane == 0) mine[r.warp] = v;
  r.meet();
  float all = mine[0];
  for (int i = 1; i < r.p.warps; ++i) {
    if constexpr (MAX) all = larger(all, mine[i]);
    else all += mine[i];
  }
  return all;
}

// K: chunks of a warp; h and z stay in registers.  SUM: h is not x; DROP: with dropout.
template <typename T, int K, int QUANT, bool SUM, bool DROP>
__global__ void __launch_bounds__(256, 2) k_rms_forward_ring(const Rms p, const RmsRing q) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int gave_up;
  constexpr int kInputs = SUM ? 2 : 1;
  Ring<kInputs> r = ring_begin<kInputs>(p, q, smem, &gave_up);
  r.in[0] = {p.x, p.x_row * (long long)sizeof(T)};
  if constexpr (SUM) r.in[1] = {p.residual, p.residual_row * (long long)sizeof(T)};
  const bool asks = r.warp == 0 && r.lane == 0;
  if (asks)
    for (int n = 0; n < q.stages; ++n) r.ask(n);
  DropKey key{};
  if constexpr (DROP) key = drop_key(p.drop);
  const uint32_t weight = tc::smem_of(smem + q.weight_at);
  const int sub = r.lane / q.lanes, first_col = (r.lane - sub * q.lanes) * 8 + r.warp * kChunk;
  const int step = p.warps * kChunk;
  const bool two = SUM && p.residual;
  unsigned s = 0;
  long long n = 0;
  for (long long u = r.first; u < r.units; u += r.step, ++n) {
    const long long row = u * q.rows + sub;
    const bool on = row < p.rows && sub < q.rows;
    const uint32_t x = tc::smem_of(r.place(int(s), 0)) + sub * q.row_bytes, res = x + q.unit_bytes;
    const unsigned long long at = (unsigned long long)row * p.d;
    r.await(n);
    Eight<T> h[K];
    float2 sq = both(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = first_col + k * step;
      if (!on || c >= p.d) continue;
      h[k].load_shared(x + c * sizeof(T));
      float2 v[4];
      h[k].get(v);
      if constexpr (SUM) {
        if constexpr (DROP) drop_pairs(v, (at + c) >> 3, key, p.drop);
        if (two) {
          Eight<T> a;
          a.load_shared(res + c * sizeof(T));
          float2 w[4];
          a.get(w);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = add2(v[i], w[i]);
        }
        h[k].set(v);
        h[k].store(static_cast<T*>(p.h) + at + c);
        h[k].get(v);
      }
      float2 t = mul2(v[0], v[0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) t = fma2(v[i], v[i], t);
      sq = fma2(t, both(p.inv_d), sq);
    }
    const float rstd = rsqrtf(ring_join<false>(r, sq.x + sq.y, int(n & 1)) + p.eps);
    // every warp of the group is done with the places up to this one's
    if (asks) r.ask(n + q.stages);
    if (on && first_col == 0 && p.rstd) p.rstd[row] = rstd;
    const auto norm8 = [&](int k, int c, float2(&v)[4]) {
      h[k].get(v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], both(rstd));
      if (p.weight) {
        Eight<float> w;
        w.load_shared(weight + c * 4);
        float2 f[4];
        w.get(f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f[i]);
      }
    };
    if constexpr (QUANT == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = first_col + k * step;
        if (!on || c >= p.d) continue;
        float2 v[4];
        norm8(k, c, v);
        Eight<T> y;
        y.set(v);
        y.store(static_cast<T*>(p.y) + at + c);
      }
    } else {
      float* scales = p.scales + row * p.blocks;
      float2 z[K][4];
      float top = 0.f, one = 1.f;
      const auto max_of = [](const float2(&v)[4]) {  // of the bits of magnitudes: NaN lies above infinity
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          m = max(m, max(__float_as_uint(v[i].x) & 0x7FFFFFFFu, __float_as_uint(v[i].y) & 0x7FFFFFFFu));
        return __uint_as_float(m);
      };
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = first_col + k * step;
#pragma unroll
        for (int i = 0; i < 4; ++i) z[k][i] = both(0.f);
        if (on && c < p.d) norm8(k, c, z[k]);
        if (p.block == 0) top = larger(top, max_of(z[k]));
      }
      if (p.block == 0) {
        one = scale_of(ring_join<true>(r, top, 2 + int(n & 1)), p.most);
        if (on && first_col == 0) scales[0] = one;
      }
      const int lanes = min(p.block / 8, q.lanes);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = first_col + k * step;
        float scale = one;
        if (p.block) {  // (all lanes: the maximum of a block is exchanged between them)
          scale = scale_of(lanes_max(max_of(z[k]), lanes), p.most);
          if (on && c < p.d && c % p.block == 0) scales[c / p.block] = scale;
        }
        if (!on || c >= p.d) continue;
        const float inv = inverse_of(scale);
        uint2 o = {0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          o.x |= quantized2<QUANT == 1>(z[k][j], inv) << (16 * j);
          o.y |= quantized2<QUANT == 1>(z[k][2 + j], inv) << (16 * j);
        }
        *reinterpret_cast<uint2*>(static_cast<unsigned char*>(p.y) + at + c) = o;
      }
    }
    s = s + 1 == unsigned(q.stages) ? 0 : s + 1;
  }
  if (asks) r.end(n + q.stages);
  if (threadIdx.x == 0 && *(volatile int*)&gave_up) atomicExch(p.status, EFCP_ETIMEOUT);
}

// K: chunks of a warp; it holds their sums of the weight's gradient in registers.
template <typename T, int K, bool DROP>
__global__ void __launch_bounds__(256, 2) k_rms_backward_ring(const Rms p, const RmsRing q) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int gave_up;
  Ring<3> r = ring_begin<3>(p, q, smem, &gave_up);
  r.in[0] = {p.dy, p.dy_row * (long long)sizeof(T)};
  r.in[1] = {p.x, p.x_row * (long long)sizeof(T)};
  r.in[2] = {p.dh, p.dh_row * (long long)sizeof(T)};
  const bool asks = r.warp == 0 && r.lane == 0;
  if (asks)
    for (int n = 0; n < q.stages; ++n) r.ask(n);
  DropKey key{};
  if constexpr (DROP) key = drop_key(p.drop);
  const uint32_t weight = tc::smem_of(smem + q.weight_at);
  const int sub = r.lane / q.lanes, first_col = (r.lane - sub * q.lanes) * 8 + r.warp * kChunk;
  const int step = p.warps * kChunk;
  float2 dw[K][4];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[k][i] = both(0.f);
  const auto rstd_of = [&](long long u) {
    const long long row = u * q.rows + sub;
    return row < p.rows ? p.rstd[row] : 0.f;
  };
  const auto weight8 = [&](int c, float2(&w)[4]) {
    Eight<float> a;
    a.load_shared(weight + c * 4);
    a.get(w);
  };
  unsigned s = 0;
  long long n = 0;
  float next = rstd_of(r.first);
  for (long long u = r.first; u < r.units; u += r.step, ++n) {
    const long long row = u * q.rows + sub;
    const bool on = row < p.rows && sub < q.rows;
    const uint32_t dy = tc::smem_of(r.place(int(s), 0)) + sub * q.row_bytes, h = dy + q.unit_bytes,
                   dh = h + q.unit_bytes;
    const unsigned long long at = (unsigned long long)row * p.d;
    const float rs = next;
    next = rstd_of(u + r.step);
    r.await(n);
    Eight<T> a8[K], b8[K];
    float2 sum = both(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = first_col + k * step;
      if (!on || c >= p.d) continue;
      a8[k].load_shared(dy + c * sizeof(T));
      b8[k].load_shared(h + c * sizeof(T));
      float2 a[4], b[4];
      a8[k].get(a);
      b8[k].get(b);
      if (p.weight) {
        float2 w[4];
        weight8(c, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = mul2(a[i], w[i]);
      }
      float2 t = mul2(a[0], b[0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) t = fma2(a[i], b[i], t);
      sum = add2(sum, t);
    }
    const float m = -ring_join<false>(r, sum.x + sum.y, int(n & 1)) * p.inv_d * rs * rs;
    // every warp of the group is done with the place before this one (its last input is read below)
    if (asks && n > 0) r.ask(n - 1 + q.stages);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = first_col + k * step;
      if (!on || c >= p.d) continue;
      float2 a[4], b[4];
      a8[k].get(a);
      b8[k].get(b);
#pragma unroll
      for (int i = 0; i < 4; ++i) dw[k][i] = fma2(a[i], mul2(b[i], both(rs)), dw[k][i]);
      if (p.weight) {
        float2 w[4];
        weight8(c, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = mul2(a[i], w[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = mul2(fma2(b[i], both(m), a[i]), both(rs));
      if (p.dh) {
        Eight<T> e8;
        e8.load_shared(dh + c * sizeof(T));
        float2 e[4];
        e8.get(e);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = add2(a[i], e[i]);
      }
      Eight<T> out;
      if (p.dresidual) {
        out.set(a);
        out.store(static_cast<T*>(p.dresidual) + at + c);
      }
      if (p.dx) {
        if constexpr (DROP) drop_pairs(a, (at + c) >> 3, key, p.drop);
        out.set(a);
        out.store(static_cast<T*>(p.dx) + at + c);
      }
    }
    s = s + 1 == unsigned(q.stages) ? 0 : s + 1;
  }
  if (p.part) {
    if (q.lanes < 32) {  // the rows of a unit, one warp
#pragma unroll
      for (int i = 0; i < 4; ++i)
        for (int o = q.lanes; o < 32; o *= 2) {
          dw[0][i].x += __shfl_xor_sync(kAll, dw[0][i].x, o);
          dw[0][i].y += __shfl_xor_sync(kAll, dw[0][i].y, o);
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = first_col + k * step;
      if (sub || c >= p.d) continue;
      Eight<float> out;
      out.set(dw[k]);
      out.store(p.part + r.first * p.d + c);
    }
  }
  if (asks) r.end(n - 1 + q.stages);
  if (threadIdx.x == 0 && *(volatile int*)&gave_up) atomicExch(p.status, EFCP_ETIMEOUT);
}

template <typename T, int K>
cudaError_t rms_launch_ring_k(const Rms& p, const RmsLaunch& l) {
  const Shape s{l.blocks, unsigned(p.groups * p.warps * 32), l.smem, 0};
  const bool sum = p.h, drop = p.drop.threshold;
  switch (l.op) {
    case kRmsE4M3:
      return sum ? launch(k_rms_forward_ring<T, K, 1, true, false>, s, l.st, p, l.ring)
                 : launch(k_rms_forward_ring<T, K, 1, false, false>, s, l.st, p, l.ring);
    case kRmsInt8:
      return sum ? launch(k_rms_forward_ring<T, K, 2, true, false>, s, l.st, p, l.ring)
                 : launch(k_rms_forward_ring<T, K, 2, false, false>, s, l.st, p, l.ring);
    case kRmsForward:
      return drop  ? launch(k_rms_forward_ring<T, K, 0, true, true>, s, l.st, p, l.ring)
             : sum ? launch(k_rms_forward_ring<T, K, 0, true, false>, s, l.st, p, l.ring)
                   : launch(k_rms_forward_ring<T, K, 0, false, false>, s, l.st, p, l.ring);
    default:
      return drop ? launch(k_rms_backward_ring<T, K, true>, s, l.st, p, l.ring)
                  : launch(k_rms_backward_ring<T, K, false>, s, l.st, p, l.ring);
  }
}

template <typename T>
cudaError_t rms_launch_ring(const Rms& p, const RmsLaunch& l) {
  const cudaError_t e = l.kept == 1   ? rms_launch_ring_k<T, 1>(p, l)
                        : l.kept == 2 ? rms_launch_ring_k<T, 2>(p, l)
                                      : rms_launch_ring_k<T, 4>(p, l);
  if (e != cudaSuccess || !p.part) return e;
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
    return launch(k_dropout<T, VEC>, Shape{l.blocks, 256, 0, 0}, l.st, p);
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
  return launch(k_rms_dweight_join, Shape{unsigned((p.d + 31) / 32), 1024, 0, 0}, l.st,
                static_cast<const float*>(p.part), l.parts, p.d, p.dweight, p.param_dtype);
}

template <typename T>
cudaError_t rms_launch(const Rms& p, const RmsLaunch& l) {
  if (l.ringed) return rms_launch_ring<T>(p, l);
  return l.vec ? rms_launch_vec<T, true>(p, l) : rms_launch_vec<T, false>(p, l);
}

}  // namespace
}  // namespace efcp
