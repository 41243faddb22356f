// Rows of d elements, cut into chunks of 256 that a warp takes eight to a lane: side by side in one or two
// 16-byte accesses where every row starts on 16 bytes (VEC), else 32 apart, so that a warp's accesses still
// touch neighbouring elements.
#pragma once

#include <cuda_fp8.h>

#include "efcp_num.cuh"
#include "efcp_philox.cuh"

namespace efcp {

constexpr int kChunk = 256;
constexpr unsigned kAll = 0xFFFFFFFFu;

// column of a lane's element j in the chunk that starts at c0
template <bool VEC>
__device__ __forceinline__ int col_of(int c0, int lane, int j) {
  return VEC ? c0 + lane * 8 + j : c0 + j * 32 + lane;
}

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c0, int lane, int d, float (&v)[8]) {
  if constexpr (VEC) {
    const int col = c0 + lane * 8;
    if (col < d) {
      Pack<T, 8> a;
      const uint4* from = reinterpret_cast<const uint4*>(row + col);
#pragma unroll
      for (int i = 0; i < int(sizeof(a) / 16); ++i) reinterpret_cast<uint4*>(&a)[i] = from[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = to_f32(a.v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = c0 + j * 32 + lane;
      v[j] = col < d ? to_f32(row[col]) : 0.f;
    }
  }
}

// the same from an array whose type is known at run time
template <bool VEC>
__device__ __forceinline__ void load8_param(const void* p, int dtype, int c0, int lane, int d,
                                            float (&v)[8]) {
  if (dtype == 0) load8<float, VEC>(static_cast<const float*>(p), c0, lane, d, v);
  else if (dtype == 1)
    load8<__nv_bfloat16, VEC>(static_cast<const __nv_bfloat16*>(p), c0, lane, d, v);
  else load8<__half, VEC>(static_cast<const __half*>(p), c0, lane, d, v);
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int c0, int lane, int d, const float (&v)[8]) {
  if constexpr (VEC) {
    const int col = c0 + lane * 8;
    if (col < d) {
      Pack<T, 8> a;
#pragma unroll
      for (int j = 0; j < 8; ++j) a.v[j] = from_f32<T>(v[j]);
      uint4* to = reinterpret_cast<uint4*>(row + col);
#pragma unroll
      for (int i = 0; i < int(sizeof(a) / 16); ++i) to[i] = reinterpret_cast<const uint4*>(&a)[i];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = c0 + j * 32 + lane;
      if (col < d) row[col] = from_f32<T>(v[j]);
    }
  }
}

// Bit j: element j * 32 + lane of the chunk whose first element is `first` in the logical order stays.  Rows need not
// start on a multiple of eight: the 32 groups that begin in the chunk are spread over the lanes, with one more behind
// them.
__device__ __forceinline__ uint32_t keep8(unsigned long long first, int lane, const DropKey& key,
                                          uint32_t threshold) {
  const int s = int(first & 7);
  const uint32_t mine = drop_keep8((first >> 3) + lane, key, threshold);
  const uint32_t last = s ? drop_keep8((first >> 3) + 32, key, threshold) : 0;
  uint32_t keep = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int q = j * 32 + lane + s;
    const uint32_t other = __shfl_sync(kAll, mine, (q >> 3) & 31);
    keep |= (((q >= 256 ? last : other) >> (q & 7)) & 1u) << j;
  }
  return keep;
}

// Dropout of a lane's eight elements of that chunk.
template <bool VEC>
__device__ __forceinline__ void drop8(float (&v)[8], unsigned long long first, int lane, const DropKey& key,
                                      const Drop& drop) {
  if constexpr (VEC) {
    drop_group(v, (first >> 3) + lane, key, drop.threshold, drop.scale);
  } else {
    const uint32_t keep = keep8(first, lane, key, drop.threshold);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? v[j] * drop.scale : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ float rounded(float v) {
  return to_f32(from_f32<T>(v));
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// The larger of two magnitudes (neither negative); a NaN, whose bits lie above infinity's, wins.
__device__ __forceinline__ float larger(float a, float b) {
  return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}
// The largest over `width` neighbouring lanes (a power of two).
__device__ __forceinline__ float lanes_max(float v, int width) {
  if (width == 32) return __uint_as_float(__reduce_max_sync(kAll, __float_as_uint(v)));
  for (int o = width / 2; o; o >>= 1) v = larger(v, __shfl_xor_sync(kAll, v, o));
  return v;
}

// ------------------------------------------------------------------ 8 bits
// The scale of a block whose largest magnitude is `top`: 1 for zeros, NaN where a value is not finite.
__device__ __forceinline__ float scale_of(float top, float most) {
  if (!(top < __int_as_float(0x7F800000))) return __int_as_float(0x7FC00000);
  const float s = top / most;
  return s > 0.f ? s : 1.f;
}

// 1 / s; 0 for a scale of NaN, or one so small that the inverse would leave fp32's range.
__device__ __forceinline__ float inverse_of(float s) { return s >= 0x1p-100f ? __fdividef(1.f, s) : 0.f; }

// z / s as 8 bits, given inverse_of(s): the quotient is off by a few roundings of fp32, so a value that close to the
// border between two 8-bit ones may go either way; 0 in a block whose scale is NaN.
template <bool E4M3>
__device__ __forceinline__ unsigned quantized(float z, float s, float inv) {
  const float q = inv > 0.f ? z * inv : s > 0.f ? z / s : 0.f;
  if constexpr (E4M3) return __nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
  else return unsigned(max(-127, min(127, __float2int_rn(q)))) & 0xFFu;
}
template <bool E4M3>
__device__ __forceinline__ uint2 quantized8(const float2 (&z)[4], float s, float inv) {
  uint2 o = {0, 0};
  if (inv > 0.f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 q = mul2(z[j], both(inv));
      unsigned w;
      if constexpr (E4M3) {
        w = __nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, __NV_E4M3);
      } else {  // (|q| is at most 127 and a few roundings)
        w = (unsigned(__float2int_rn(q.x)) & 0xFFu) | (unsigned(__float2int_rn(q.y)) & 0xFFu) << 8;
      }
      (j < 2 ? o.x : o.y) |= w << (16 * (j & 1));
    }
  } else if (s > 0.f) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      (j < 2 ? o.x : o.y) |= (quantized<E4M3>(z[j].x, s, 0.f) | quantized<E4M3>(z[j].y, s, 0.f) << 8) << (16 * (j & 1));
  }
  return o;
}

}  // namespace efcp
