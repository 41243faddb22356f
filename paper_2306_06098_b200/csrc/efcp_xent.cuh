// Softmax cross entropy of a linear layer over a vocabulary (the formulas stand in include/efcp.h), in products of
// tiles on the fifth-generation tensor cores.  The logits never reach memory: a tile of them is turned into the rows'
// largest value and sum of exponentials, and in the backward pass, computed once more for a piece of the vocabulary
// at a time, into their gradient, which the two products behind it read.
//
// A block holds one SM: a warp that copies tiles of both operands into a ring in shared memory, a warp that issues the
// products into one of two accumulators in tensor memory, and eight warps that work on the other accumulator.
// Every wait is bounded; when one runs out the block ends, and the status tells of it.
//
// fp32 values are held as three bfloat16 ones (8 bits of the significand each), of whose nine products the six
// largest are added up, the small ones first; what is left out is below 2^-24 of the result.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_num.cuh"
#include "efcp_rows.cuh"
#include "efcp_tc.cuh"
#include "efcp_xent.h"

namespace efcp {
namespace {

constexpr int kStages = 4;
constexpr int kOutWarps = 8, kXentThreads = (kOutWarps + 2) * 32;
constexpr uint32_t kBoxBytes = 64 * 128;
constexpr uint32_t kABytes = kXentRows / 64 * kBoxBytes, kBBytes = kXentCols / 64 * kBoxBytes;
constexpr size_t kXentSmem = kStages * (kABytes + kBBytes) + 1024;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
using Operand = std::conditional_t<std::is_same_v<T, __half>, __half, __nv_bfloat16>;

__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 32 values to T, `valid` of them
template <typename T>
__device__ __forceinline__ void store32(T* to, int valid, bool vec, const float (&v)[32]) {
  constexpr int kPer = 16 / sizeof(T);
  if (vec && valid >= 32) {
#pragma unroll
    for (int i = 0; i < 32; i += kPer) {
      Pack<T, kPer> a;
#pragma unroll
      for (int j = 0; j < kPer; ++j) a.v[j] = from_f32<T>(v[i + j]);
      *reinterpret_cast<uint4*>(to + i) = *reinterpret_cast<const uint4*>(&a);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < valid) to[i] = from_f32<T>(v[i]);
  }
}

// x as up to three values of O whose sum it is
template <typename O, int PLANES>
__device__ __forceinline__ void split(float x, O (&v)[PLANES]) {
#pragma unroll
  for (int i = 0; i < PLANES; ++i) {
    v[i] = from_f32<O>(x);
    x -= to_f32(v[i]);
  }
}

template <int MODE, typename T>
__global__ void __launch_bounds__(kXentThreads, 1) k_xent(const __grid_constant__ XentGemm p) {
  using O = Operand<T>;
  constexpr bool kAMn = MODE == kXentWeight, kBMn = MODE >= kXentHidden;
  constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 1, kPairs = kPlanes == 3 ? 6 : 1;
  extern __shared__ unsigned char ring_[];
  __shared__ alignas(8) uint64_t bars[2 * kStages + 5];
  __shared__ uint32_t tmem_at;
  __shared__ int gave_up_;
  volatile int* gave_up = &gave_up_;
  const uint32_t ring = (tc::smem_of(ring_) + 1023) & ~1023u;
  const uint32_t full = tc::smem_of(bars), empty = full + 8 * kStages, done = empty + 8 * kStages,
                 taken = done + 16, drained = taken + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    gave_up_ = 0;
    for (int i = 0; i < kStages; ++i) {
      tc::bar_init(full + 8 * i, 1);
      tc::bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::bar_init(done + 8 * i, 1);
      tc::bar_init(taken + 8 * i, kOutWarps);
    }
    tc::bar_init(drained, 1);
    tc::bar_init_fence();
  }
  if (warp == kOutWarps) {
    tc::tmem_alloc(tc::smem_of(&tmem_at), 512);
    if (lane == 0) {
      tc::prefetch_map(&p.a);
      tc::prefetch_map(&p.b);
    }
  }
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  take_turn();
  const uint32_t tmem = tmem_at;
  const int count = *p.count;
  const int row_tiles = p.row_tiles >= 0 ? p.row_tiles : (count + kXentRows - 1) / kXentRows;
  const int depth = ((p.depth >= 0 ? p.depth : count) + kXentDepth - 1) / kXentDepth;
  const int steps = depth * kPairs;
  const long long tiles = (long long)row_tiles * p.col_tiles;

  if (warp == kOutWarps) {
    if (lane == 0) {
      // copies: rows first, so that a tile of the other operand serves many blocks at the same time
      const uint32_t bytes = kABytes + uint32_t(p.col_tile / 64) * kBoxBytes;
      unsigned n = 0;  // steps so far
      bool ok = true;
      for (long long t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
        const int tc_ = int(t / row_tiles), m0 = int(t - (long long)tc_ * row_tiles) * kXentRows,
                  n0 = tc_ * p.col_tile;
        const int an = m0, bn = MODE == kXentGrad ? p.v0 + n0 : n0;
        const int bk = MODE == kXentHidden ? p.v0 : 0;
        for (int i = 0; i < steps && ok; ++i, ++n) {
          const int pair = kPairs == 1 ? 0 : i / depth, k = (i - pair * depth) * kXentDepth;
          // planes of the pairs: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
          const int pa = kPairs == 1 ? 0 : (0x001102 >> (4 * pair)) & 15;
          const int pb = kPairs == 1 ? 0 : (0x010120 >> (4 * pair)) & 15;
          const unsigned s = n % kStages;
          ok = tc::bar_wait(empty + 8 * s, (n / kStages + 1) & 1, gave_up);
          if (!ok) break;
          const uint32_t bar = full + 8 * s, at = ring + s * (kABytes + kBBytes);
          tc::bar_expect(bar, bytes);
#pragma unroll
          for (int j = 0; j < kXentRows / 64; ++j)
            tc::load_box(&p.a, at + j * kBoxBytes, bar, kAMn ? an + 64 * j : k, kAMn ? k : an + 64 * j, pa);
          for (int j = 0; j < p.col_tile / 64; ++j)
            tc::load_box(&p.b, at + kABytes + j * kBoxBytes, bar, kBMn ? bn + 64 * j : k,
                         kBMn ? bk + k : bn + 64 * j, pb);
        }
      }
      if (!ok)  // nothing may land in shared memory that the block has left
        for (unsigned i = n < kStages ? 0 : n - kStages; i < n; ++i)
          (void)tc::bar_wait(full + 8 * (i % kStages), (i / kStages) & 1, gave_up, tc::kDrainNs);
    }
    __syncwarp();
  } else if (warp == kOutWarps + 1) {
    if (lane == 0) {
      const uint32_t ins = tc::instruction(std::is_same_v<O, __nv_bfloat16>, kXentRows, p.col_tile, kAMn, kBMn);
      unsigned n = 0, turn = 0;
      bool ok = true;
      for (long long t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++turn) {
        const unsigned buf = turn & 1;
        ok = tc::bar_wait(taken + 8 * buf, (turn / 2 + 1) & 1, gave_up);
        if (!ok) break;
        tc::fence_after();
        for (int i = 0; i < steps; ++i, ++n) {
          const unsigned s = n % kStages;
          ok = tc::bar_wait(full + 8 * s, (n / kStages) & 1, gave_up);
          if (!ok) break;
          tc::fence_after();
          const uint32_t a = ring + s * (kABytes + kBBytes), b = a + kABytes;
#pragma unroll
          for (int k = 0; k < kXentDepth / 16; ++k)
            tc::mma(tmem + buf * kXentCols, tc::operand(a + k * (kAMn ? 2048 : 32), kBoxBytes),
                    tc::operand(b + k * (kBMn ? 2048 : 32), kBoxBytes), ins, i > 0 || k > 0);
          tc::commit(empty + 8 * s);
        }
        if (ok) tc::commit(done + 8 * buf);
      }
      if (!ok) {  // the products under way end before the tensor memory is given back
        tc::commit(drained);
        (void)tc::bar_wait(drained, 0, gave_up, tc::kDrainNs);
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, half = warp >> 2, cols = p.col_tile / 2;
    unsigned turn = 0;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x, ++turn) {
      const unsigned buf = turn & 1;
      const int tc_ = int(t / row_tiles), m0 = int(t - (long long)tc_ * row_tiles) * kXentRows;
      const int row = m0 + quarter * 32 + lane, n0 = tc_ * p.col_tile + half * cols;
      int target = -1;
      float lse = 0.f, coef = 0.f, back = 1.f;
      if constexpr (MODE == kXentStats || MODE == kXentGrad) target = p.target[row];
      if constexpr (MODE == kXentGrad) {
        lse = p.lse[row];
        coef = p.coef[row];
      }
      if constexpr (MODE >= kXentHidden) back = p.scale[1];
      if (!__all_sync(kAll, tc::bar_wait(done + 8 * buf, (turn / 2) & 1, gave_up))) break;
      tc::fence_after();
      const uint32_t at = tmem + buf * kXentCols + half * cols + (uint32_t(quarter * 32) << 16);
      float top = -INFINITY, total = 0.f;
      for (int c = 0; c < cols; c += 32) {
        float v[32];
        __syncwarp();
        tc::tmem_load32(at + c, v);
        const int col = n0 + c;
        if constexpr (MODE == kXentStats) {
          const int valid = p.vocab - col;
          if (valid <= 0) continue;
          const int hit = target - col;
          if (hit >= 0 && hit < 32) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) x = i == hit ? v[i] : x;
            p.target_logit[row] = x;
          }
          if (valid < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = i < valid ? v[i] : -INFINITY;
          }
          float m = top;
#pragma unroll
          for (int i = 0; i < 32; ++i) m = fmaxf(m, v[i]);
          const float base = m == -INFINITY ? 0.f : m;
          total *= pow2((top - base) * kLog2e);
          top = m;
          float s[4] = {};
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i & 3] += pow2((v[i] - base) * kLog2e);
          total += (s[0] + s[1]) + (s[2] + s[3]);
        } else if constexpr (MODE == kXentGrad) {
          if (col >= int(p.g_row)) continue;
          const int hit = target - (p.v0 + col), valid = row < count ? min(p.piece, p.vocab - p.v0) - col : 0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = pow2((v[i] - lse) * kLog2e) - (i == hit ? 1.f : 0.f);
            v[i] = i < valid ? x * coef : 0.f;
          }
          O* to = static_cast<O*>(p.g) + (long long)row * p.g_row + col;
          if constexpr (kPlanes == 1) {
            store32<O>(to, 32, true, v);
          } else {
#pragma unroll
            for (int plane = 0; plane < kPlanes; ++plane) {
              store32<O>(to + plane * p.g_plane, 32, true, v);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] -= rounded<O>(v[i]);
            }
          }
        } else if constexpr (MODE == kXentHidden) {
          const int valid = p.d - col;
          if (row >= count || valid <= 0) continue;
          float* sum = p.sum + row * p.sum_row + col;  // (rows of whole 32s)
          if (!p.first) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float4 o = *reinterpret_cast<const float4*>(sum + i);
              v[i] += o.x; v[i + 1] += o.y; v[i + 2] += o.z; v[i + 3] += o.w;
            }
          }
          if (p.last) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= back;
            store32<T>(static_cast<T*>(p.out) + (long long)p.order[row] * p.out_row + col, valid, p.vec_out, v);
          } else {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<float4*>(sum + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          }
        } else {
          const int valid = p.d - col;
          if (row >= min(p.piece, p.vocab - p.v0) || valid <= 0) continue;
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = steps ? v[i] * back : 0.f;
          store32<T>(static_cast<T*>(p.out) + (long long)(p.v0 + row) * p.out_row + col, valid, p.vec_out, v);
        }
      }
      if constexpr (MODE == kXentStats)
        p.part[(long long)row * p.parts + tc_ * 2 + half] = make_float2(top, total);
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::bar_arrive(taken + 8 * buf);
    }
  }
  tc::fence_before();
  __syncthreads();
  if (warp == kOutWarps) tc::tmem_free(tmem, 512);
  if (threadIdx.x == 0 && gave_up_) atomicExch(p.status, EFCP_ETIMEOUT);
}

// Sum of v over the threads before this one of a block of 1024, and over all.
__device__ __forceinline__ int block_before(int v, int* all) {
  __shared__ int part[33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = v;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int other = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += other;
  }
  if (lane == 31) part[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int w = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int other = __shfl_up_sync(kAll, w, o);
      if (lane >= o) w += other;
    }
    part[lane] = w;
  }
  __syncthreads();
  *all = part[31];
  return sum - v + (warp ? part[warp - 1] : 0);
}

// One block: which tokens have a target, in order; backward also the factors on their gradients, times a power of two
// that brings the largest near 1 (near 2^14 for fp16, whose probabilities would vanish otherwise).
template <bool HALF>
__global__ void __launch_bounds__(1024) k_xent_select(const XentPrep p, bool backward) {
  take_turn();
  __shared__ unsigned most;
  const long long per = (p.tokens + 1023) / 1024, lo = threadIdx.x * per, hi = min(p.tokens, lo + per);
  if (threadIdx.x == 0) most = 0;
  int mine = 0, all;
  for (long long i = lo; i < hi; ++i) mine += p.targets[i] != p.ignore;
  int at = block_before(mine, &all);
  const float mean = p.reduction == 1 ? 1.f / float(all) : 1.f;
  float big = 0.f;
  for (long long i = lo; i < hi; ++i) {
    const long long t = p.targets[i];
    if (t == p.ignore) continue;
    const bool in = t >= 0 && t < p.vocab;
    p.order[at] = int(i);
    p.target[at] = in ? int(t) : -1;
    if (backward) {
      const float g = p.grad[p.reduction ? 0 : i * p.grad_step] * mean;
      p.coef[at] = in ? g : __int_as_float(0x7FC00000);
      p.lse[at] = p.lse_in[i];
      if (fabsf(g) < INFINITY) big = fmaxf(big, fabsf(g));
    }
    ++at;
  }
  for (int i = all + threadIdx.x; i < (all + kXentRows - 1) / kXentRows * kXentRows; i += 1024) {
    p.target[i] = -1;
    if (backward) p.coef[i] = p.lse[i] = 0.f;
  }
  if (threadIdx.x == 0) *p.count = all;
  if (!backward) return;
  atomicMax(&most, __float_as_uint(big));  // (of values that are not negative the bits are in order)
  __syncthreads();
  big = __uint_as_float(most);
  const int e = big > 0.f ? max(-100, min(100, ilogbf(big))) : 0;
  const float up = scalbnf(1.f, (HALF ? 14 : 0) - e);
  if (threadIdx.x == 0) {
    p.scale[0] = up;
    p.scale[1] = scalbnf(1.f, e - (HALF ? 14 : 0));
  }
  for (int i = threadIdx.x; i < all; i += 1024) p.coef[i] *= up;
}

// Rows of H that have a target, one behind the other (and zeros up to whole tiles), as the copies of tiles want them;
// what belongs to the other tokens becomes zero.  A warp takes a row.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_gather(const XentPrep p) {
  take_turn();
  using O = Operand<T>;
  constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 1;
  const int lane = threadIdx.x & 31, count = *p.count;
  const long long padded = (count + kXentRows - 1) / kXentRows * kXentRows;
  const long long warps = (long long)gridDim.x * 8, first = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  for (long long i = first; i < padded; i += warps) {
    const T* from = static_cast<const T*>(p.hidden) + (i < count ? (long long)p.order[i] * p.hidden_row : 0);
    O* to = static_cast<O*>(p.hidden_packed) + i * p.packed_row;
    const bool vec = kPlanes == 1 && reinterpret_cast<uintptr_t>(from) % 16 == 0 && p.d % 8 == 0;
    if (vec) {
      for (int c = lane * 8; c < p.d; c += 256)
        *reinterpret_cast<uint4*>(to + c) =
            i < count ? *reinterpret_cast<const uint4*>(from + c) : make_uint4(0, 0, 0, 0);
    } else {
      for (int c = lane; c < p.d; c += 32) {
        O v[kPlanes];
        split<O, kPlanes>(i < count ? to_f32(from[c]) : 0.f, v);
#pragma unroll
        for (int k = 0; k < kPlanes; ++k) to[k * p.hidden_plane + c] = v[k];
      }
    }
  }
  for (long long i = first; i < p.tokens; i += warps) {
    if (p.targets[i] != p.ignore) continue;
    if (lane == 0 && p.losses && !p.reduction) p.losses[i] = 0.f;
    if (lane == 0 && p.lse_out) p.lse_out[i] = 0.f;
    if (p.dhidden)
      for (int c = lane; c < p.d; c += 32) static_cast<T*>(p.dhidden)[i * p.d + c] = from_f32<T>(0.f);
  }
}

// W as the copies of tiles want it, where it does not lie so.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_pack(const XentPrep p) {
  take_turn();
  using O = Operand<T>;
  constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 1;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * 8;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < p.vocab; i += warps) {
    const T* from = static_cast<const T*>(p.weight) + i * p.weight_row;
    O* to = static_cast<O*>(p.weight_packed) + i * p.packed_row;
    for (int c = lane; c < p.d; c += 32) {
      O v[kPlanes];
      split<O, kPlanes>(to_f32(from[c]), v);
#pragma unroll
      for (int k = 0; k < kPlanes; ++k) to[k * p.weight_plane + c] = v[k];
    }
  }
}

template <int MODE, typename T>
cudaError_t xent_launch(const XentGemm& p, unsigned blocks, cudaStream_t st) {
  const auto kern = k_xent<MODE, T>;
  // (the same value every time: a kernel's limit belongs to the device, not to this launch)
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kXentSmem));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kXentThreads);
  cfg.dynamicSmemBytes = kXentSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <typename T>
cudaError_t xent_gemm(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st) {
  switch (mode) {
    case kXentStats: return xent_launch<kXentStats, T>(p, blocks, st);
    case kXentGrad: return xent_launch<kXentGrad, T>(p, blocks, st);
    case kXentHidden: return xent_launch<kXentHidden, T>(p, blocks, st);
    default: return xent_launch<kXentWeight, T>(p, blocks, st);
  }
}

template <typename T>
cudaError_t xent_prepare(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  cudaError_t e = launch(k_xent_select<std::is_same_v<T, __half>>, Shape{1, 1024, 0, 0}, st, p, backward);
  if (e != cudaSuccess) return e;
  const auto blocks = [&](long long rows) {
    return unsigned(rows / 8 + 1 < 8ll * sms ? rows / 8 + 1 : 8ll * sms);
  };
  e = launch(k_xent_gather<T>, Shape{blocks(p.tokens + kXentRows), 256, 0, 0}, st, p);
  if (e != cudaSuccess || !p.weight) return e;
  return launch(k_xent_pack<T>, Shape{blocks(p.vocab), 256, 0, 0}, st, p);
}

}  // namespace
}  // namespace efcp
