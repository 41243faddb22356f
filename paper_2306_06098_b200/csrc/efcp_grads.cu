// The gradients of a model as a list of tensors: global norm, clipping, and the gather into the
// flat fp32 vector that the optimizer step reads (see include/efcp.h).
//
// All three are streams over memory with a handful of operations per element: HBM bounds them when
// the list is large, the launch when it is small.  The list travels in the kernel's parameters (up to
// 32 KB of constant memory: no copy to wait for, no host buffer that has to outlive the
// call).  It is cut into chunks of 32 KB that the thread blocks take in turn, so that one
// large matrix and hundreds of short vectors both keep every SM busy (smaller chunks when there are too
// few of them for that; a contiguous range per block instead took 41 us in place of 37 for the
// norm below, and 188 in place of 157 for the gather).
//
// Measured on a B200 (copy rate 6.56 TB/s): norm of a BERT-base in bf16 and fp32 vectors, 219 MB, 37 us,
// 5.9 TB/s; clipping ResNet-18's 47 MB in place 28 us, its norm and the factor in two launches (11 where it is in L2
// already); the clipped gather of BERT-base from bf16 157 us, 876 MB with the norm's read, 5.6 TB/s; of 301 ragged
// fp16 tensors 41 us; norm of a ResNet-20 6.0 us, its clipped gather from channels-last gradients 9.7 us.  From fp32
// gradients one after another, not clipped: ResNet-18 13.9 us, BERT-base 146 us, 6.0 TB/s.
#include "efcp.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "efcp_common.cuh"
#include "efcp_device.h"
#include "efcp_launch.cuh"
#include "efcp_num.cuh"

namespace efcp {
namespace {

constexpr int kGrThreads = 256;
constexpr int kGrBlocksPerSM = 8;
constexpr int kGrMaxBlocks = 4096;    // partial sums the workspace has room for
constexpr int kGrChunkLog = 15;     // 32 KB of the source: 128 bytes per thread
constexpr int kGrChunkLogMin = 11;  // 2 KB

// A tensor's layout when its elements do not lie one after another: up to four merged
// dimensions, [0] running fastest in the flat vector.
struct Geom {
  long long size[3];  // of dimensions 0..2 (dimension 3 is what is left)
  long long stride[4];
  // n / size[k] = n * mul[k] >> shift[k] for n < 2^31
  unsigned mul[3];
  unsigned char shift[3];
};

// What a launch works on.  first[i] is the number of the first chunk of tensor i.  M: how many tensors
// may need a Geom; with 0 the kernels leave the code for them out, which takes twice the registers.
template <int N, int M>
struct Table {
  static constexpr int kN = N, kM = M;
  const void* ptr[N];
  long long numel[N];
  long long dst[N];  // position in the flat vector
  Geom geom[M > 0 ? M : 1];
  unsigned first[N + 1];
  int n, chunk_log;
  short shape[N];  // index into geom, -1: one after another
  unsigned char dtype[N];
};

struct Work {
  double sumsq;       // of the list, complete after the last launch of the norm
  unsigned arrived;   // blocks that have stored their partial sum; wraps to zero
  unsigned pad;
  double part[kGrMaxBlocks];
};

// ------------------------------------------------------------------ device
__device__ __forceinline__ int chunk_elems(int chunk_log, int dtype) {
  return 1 << (chunk_log - (dtype == EFCP_F32 ? 2 : 1));
}

// The tensor that chunk c belongs to: the last i with first[i] <= c.
template <class Tab>
__device__ __forceinline__ int find_tensor(const Tab& tab, unsigned c) {
  int lo = 0, hi = tab.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tab.first[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Position of element e of a strided tensor.
__device__ __forceinline__ long long strided_pos(const Geom& g, long long e, bool small) {
  long long pos = 0;
  if (small) {  // fewer than 2^31 elements
    unsigned r = unsigned(e);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const unsigned q = unsigned((unsigned long long)r * g.mul[k] >> g.shift[k]);
      pos += (long long)(r - q * unsigned(g.size[k])) * g.stride[k];
      r = q;
    }
    return pos + (long long)r * g.stride[3];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const long long q = e / g.size[k];
    pos += (e - q * g.size[k]) * g.stride[k];
    e = q;
  }
  return pos + e * g.stride[3];
}

// fp32 sums of squares are good to a few 2^-24 as long as they neither overflow nor vanish.
__device__ __forceinline__ bool in_range(float s) { return s > 1e-28f && s < 1e37f; }

// The squares of N values added to t, two products to an instruction.
template <int N>
__device__ __forceinline__ void add_squares(const float (&v)[N], float2& t) {
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    const float2 x = make_float2(v[j], v[j + 1]);
    t = __ffma2_rn(x, x, t);
  }
}

template <int N>
__device__ __forceinline__ double sumsq_wide(const float (&v)[N]) {
  double d = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) d = fma(double(v[j]), double(v[j]), d);
  return d;
}

template <typename T, int V>
__device__ __forceinline__ double sumsq_of(const Pack<T, V>& a) {
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = to_f32(a.v[j]);
  float2 t = make_float2(0.f, 0.f);
  add_squares(v, t);
  const float s = t.x + t.y;
  return in_range(s) ? double(s) : sumsq_wide(v);
}

// The bits of an access's values, without their signs, joined: 0 where all are zeros.
template <typename T, int V>
__device__ __forceinline__ unsigned bits_of(const Pack<T, V>& a) {
  static_assert(sizeof(a) == 16, "four words");
  const uint4 w = *reinterpret_cast<const uint4*>(&a);
  return (w.x | w.y | w.z | w.w) & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
}

template <typename T>
__device__ __forceinline__ double chunk_sumsq(const T* p, int len) {
  constexpr int V = 16 / int(sizeof(T)), U = 4;
  using P = Pack<T, V>;
  // elements before the first 16-byte boundary
  const int skew = int((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
  const int head = min(len, skew ? V - skew : 0);
  const int nv = (len - head) / V;
  const P* q = reinterpret_cast<const P*>(p + head);
  double acc = 0.0;
  const int rest = len - head - nv * V;  // the ends: fewer than 2 V elements
  if (int(threadIdx.x) < head + rest) {
    const int k = int(threadIdx.x) < head ? int(threadIdx.x) : nv * V + int(threadIdx.x);
    const double x = double(to_f32(p[k]));
    acc += x * x;
  }
  int i = threadIdx.x;
  for (; i + (U - 1) * kGrThreads < nv; i += U * kGrThreads) {
    P a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = q[i + u * kGrThreads];
    // four sums of at most 8 products each
    float2 t[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    unsigned bits = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      bits |= bits_of(a[u]);
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = to_f32(a[u].v[j]);
      add_squares(v, t[u & 1]);
    }
    const float s = (t[0].x + t[0].y) + (t[1].x + t[1].y);
    // zeros are common (an embedding's rows without a token)
    if (in_range(s) | (bits == 0)) {
      acc += double(s);
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u) acc += sumsq_of(q[i + u * kGrThreads]);
    }
  }
#pragma unroll 1
  for (; i < nv; i += kGrThreads) acc += sumsq_of(q[i]);
  return acc;
}

template <typename T>
__device__ double chunk_sumsq_strided(const T* p, const Geom& g, long long begin, int len,
                                      bool small) {
  double acc = 0.0;
#pragma unroll 2
  for (int i = threadIdx.x; i < len; i += kGrThreads) {
    const double x = double(to_f32(p[strided_pos(g, begin + i, small)]));
    acc += x * x;
  }
  return acc;
}

// The sum over all blocks of a launch, added to `sumsq` (or stored there by the first launch of a
// list) by the block that arrives last; the partial sums are added in a fixed order.  Returns true in that
// block's thread 0.
__device__ bool finish_sum(double acc, Work* ws, bool first_launch) {
  __shared__ double sm[32];
  __shared__ bool last;
  acc = block_sum(acc, sm);
  if (threadIdx.x == 0) {
    ws->part[blockIdx.x] = acc;
    __threadfence();
    last = atomicInc(&ws->arrived, gridDim.x - 1) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return false;
  __threadfence();
  double s = 0.0;
  for (unsigned i = threadIdx.x; i < gridDim.x; i += kGrThreads) s += __ldcg(&ws->part[i]);
  s = block_sum(s, sm);
  if (threadIdx.x != 0) return false;
  ws->sumsq = first_launch ? s : ws->sumsq + s;
  return true;
}

// f = scale * min(1, max_norm / N), N = scale * sqrt(sumsq); scale when N is not finite.
__device__ __forceinline__ float factor_of(const Work* ws, double max_norm, double scale) {
  const double norm = scale * sqrt(ws->sumsq);
  return float(norm > max_norm && isfinite(norm) ? scale * (max_norm / norm) : scale);
}

template <class Tab>
__global__ void __launch_bounds__(kGrThreads, Tab::kM > 0 ? 4 : kGrBlocksPerSM)
    k_grads_sumsq(const __grid_constant__ Tab tab, Work* ws, bool first_launch, double scale,
                  float* norm) {
  take_turn();
  double acc = 0.0;
  const unsigned total = tab.first[tab.n];
  for (unsigned c = blockIdx.x; c < total; c += gridDim.x) {
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(tab.chunk_log, dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = Tab::kM > 0 ? tab.shape[i] : -1;
    if (Tab::kM == 0 || g < 0) {
      if (dtype == EFCP_F32)
        acc += chunk_sumsq(static_cast<const float*>(tab.ptr[i]) + begin, len);
      else if (dtype == EFCP_BF16)
        acc += chunk_sumsq(static_cast<const __nv_bfloat16*>(tab.ptr[i]) + begin, len);
      else
        acc += chunk_sumsq(static_cast<const __half*>(tab.ptr[i]) + begin, len);
    } else {
      const bool small = tab.numel[i] < (1ll << 31);
      if (dtype == EFCP_F32)
        acc += chunk_sumsq_strided(static_cast<const float*>(tab.ptr[i]), tab.geom[g], begin, len,
                                   small);
      else if (dtype == EFCP_BF16)
        acc += chunk_sumsq_strided(static_cast<const __nv_bfloat16*>(tab.ptr[i]), tab.geom[g],
                                   begin, len, small);
      else
        acc += chunk_sumsq_strided(static_cast<const __half*>(tab.ptr[i]), tab.geom[g], begin, len,
                                   small);
    }
  }
  if (finish_sum(acc, ws, first_launch) && norm) *norm = float(scale * sqrt(ws->sumsq));
}

template <typename T>
__device__ __forceinline__ void chunk_scale(T* p, int len, float f) {
  constexpr int V = 16 / int(sizeof(T));
  using P = Pack<T, V>;
  const int skew = int((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
  const int head = min(len, skew ? V - skew : 0);
  const int nv = (len - head) / V;
  P* q = reinterpret_cast<P*>(p + head);
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += kGrThreads) {
    P a = q[i];
#pragma unroll
    for (int j = 0; j < V; ++j) a.v[j] = from_f32<T>(to_f32(a.v[j]) * f);
    q[i] = a;
  }
  const int rest = len - head - nv * V;
  if (int(threadIdx.x) < head + rest) {
    const int i = int(threadIdx.x) < head ? int(threadIdx.x) : nv * V + int(threadIdx.x);
    p[i] = from_f32<T>(to_f32(p[i]) * f);
  }
}

template <typename T>
__device__ void chunk_scale_strided(T* p, const Geom& g, long long begin, int len, bool small,
                                    float f) {
  for (int i = threadIdx.x; i < len; i += kGrThreads) {
    T* q = p + strided_pos(g, begin + i, small);
    *q = from_f32<T>(to_f32(*q) * f);
  }
}

// The chunks run from the last to the first: the norm has just read them from the first to the
// last, and what it read last is still in L2.
template <class Tab>
__global__ void __launch_bounds__(kGrThreads, Tab::kM > 0 ? 4 : kGrBlocksPerSM)
    k_grads_scale(const __grid_constant__ Tab tab, const Work* ws, double max_norm, double scale) {
  take_turn();
  const float f = factor_of(ws, max_norm, scale);
  if (f == 1.f) return;
  const unsigned total = tab.first[tab.n];
  for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
    const unsigned c = total - 1 - b;
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(tab.chunk_log, dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = Tab::kM > 0 ? tab.shape[i] : -1;
    void* p = const_cast<void*>(tab.ptr[i]);
    const bool small = tab.numel[i] < (1ll << 31);
    if (dtype == EFCP_F32) {
      if (Tab::kM == 0 || g < 0) chunk_scale(static_cast<float*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<float*>(p), tab.geom[g], begin, len, small, f);
    } else if (dtype == EFCP_BF16) {
      if (Tab::kM == 0 || g < 0) chunk_scale(static_cast<__nv_bfloat16*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<__nv_bfloat16*>(p), tab.geom[g], begin, len, small, f);
    } else {
      if (Tab::kM == 0 || g < 0) chunk_scale(static_cast<__half*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<__half*>(p), tab.geom[g], begin, len, small, f);
    }
  }
}

// v f, or v itself when f is 1: the select is on the bits, so that a copy keeps every bit of a NaN.
__device__ __forceinline__ float scaled(float v, float f) {
  return __uint_as_float(f == 1.f ? __float_as_uint(v) : __float_as_uint(__fmul_rn(v, f)));
}

// One chunk into the flat vector; with ACC its sum of squares is returned.  A thread stores four
// elements at a time, at 16-byte boundaries of the flat vector; it loads them by one access where the
// source is aligned to that, and one by one, out of L1, where it is not (cutting them out of two
// aligned accesses was slower: 45 us against 42 for the 301 ragged fp16 tensors).
// U: such stores under way at a time.
template <typename T, bool ACC, int U, class Load>
__device__ __forceinline__ double gather_by_fours(float* dst, int len, float f, Load load) {
  const int skew = int((reinterpret_cast<uintptr_t>(dst) & 15) / 4);
  const int head = min(len, skew ? 4 - skew : 0);
  const int nv = (len - head) / 4;
  float4* out = reinterpret_cast<float4*>(dst + head);
  double acc = 0.0;
  const auto put = [&](int i, const Pack<T, 4>& a) {
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = to_f32(a.v[j]);
    if (ACC) acc += sumsq_of(a);
    out[i] = make_float4(scaled(v[0], f), scaled(v[1], f), scaled(v[2], f), scaled(v[3], f));
  };
  int i = threadIdx.x;
  if (U > 1) {
    for (; i + (U - 1) * kGrThreads < nv; i += U * kGrThreads) {
      Pack<T, 4> a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] = load.four(head + 4 * (i + u * kGrThreads));
#pragma unroll
      for (int u = 0; u < U; ++u) put(i + u * kGrThreads, a[u]);
    }
  }
#pragma unroll 1
  for (; i < nv; i += kGrThreads) put(i, load.four(head + 4 * i));
  const int rest = len - head - nv * 4;  // the ends: fewer than 8 elements
  if (int(threadIdx.x) < head + rest) {
    const int k = int(threadIdx.x) < head ? int(threadIdx.x) : nv * 4 + int(threadIdx.x);
    const float v = to_f32(load.one(k));
    if (ACC) acc += double(v) * double(v);
    dst[k] = scaled(v, f);
  }
  return acc;
}

template <typename T>
struct LoadAligned {
  const T* p;
  __device__ __forceinline__ Pack<T, 4> four(int i) const {
    return *reinterpret_cast<const Pack<T, 4>*>(p + i);
  }
  __device__ __forceinline__ T one(int i) const { return p[i]; }
};
template <typename T>
struct LoadSingly {
  const T* p;
  __device__ __forceinline__ Pack<T, 4> four(int i) const {
    Pack<T, 4> a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a.v[j] = p[i + j];
    return a;
  }
  __device__ __forceinline__ T one(int i) const { return p[i]; }
};
struct LoadZeros {
  __device__ __forceinline__ Pack<float, 4> four(int) const { return {{0.f, 0.f, 0.f, 0.f}}; }
  __device__ __forceinline__ float one(int) const { return 0.f; }
};
template <typename T>
struct LoadStrided {
  const T* p;
  const Geom& g;
  long long begin;
  bool small;
  __device__ __forceinline__ Pack<T, 4> four(int i) const {
    Pack<T, 4> a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a.v[j] = one(i + j);
    return a;
  }
  __device__ __forceinline__ T one(int i) const { return p[strided_pos(g, begin + i, small)]; }
};

template <typename T, bool ACC>
__device__ __forceinline__ double chunk_gather(const T* p, float* dst, int len, float f) {
  // (the address of the first element that goes to a 16-byte boundary of the flat vector)
  const int skew = int((reinterpret_cast<uintptr_t>(dst) & 15) / 4);
  const uintptr_t first = reinterpret_cast<uintptr_t>(p + (skew ? 4 - skew : 0));
  if (first % sizeof(Pack<T, 4>) == 0)
    return gather_by_fours<T, ACC, 4>(dst, len, f, LoadAligned<T>{p});
  return gather_by_fours<T, ACC, 2>(dst, len, f, LoadSingly<T>{p});
}

template <typename T, bool ACC>
__device__ double chunk_gather_strided(const T* p, const Geom& g, long long begin, float* dst,
                                       int len, bool small, float f) {
  return gather_by_fours<T, ACC, 1>(dst, len, f, LoadStrided<T>{p, g, begin, small});
}

// CLIP: the factor comes from the norm a launch before has left in ws.  ACC: there is no
// clipping, and the norm is taken in the same pass.
template <class Tab, bool CLIP, bool ACC>
__global__ void __launch_bounds__(kGrThreads, Tab::kM > 0 ? 4 : kGrBlocksPerSM)
    k_grads_gather(const __grid_constant__ Tab tab, float* flat, Work* ws, bool first_launch,
                   double max_norm, double scale, float* norm) {
  take_turn();
  const float f = CLIP ? factor_of(ws, max_norm, scale) : float(scale);
  const unsigned total = tab.first[tab.n];
  double acc = 0.0;
  for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
    const unsigned c = CLIP ? total - 1 - b : b;  // backwards after a norm, as k_grads_scale
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(tab.chunk_log, dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = Tab::kM > 0 ? tab.shape[i] : -1;
    const void* p = tab.ptr[i];
    float* dst = flat + tab.dst[i] + begin;
    const bool small = tab.numel[i] < (1ll << 31);
    if (!p) {
      gather_by_fours<float, false, 1>(dst, len, 1.f, LoadZeros{});
    } else if (dtype == EFCP_F32) {
      const float* q = static_cast<const float*>(p);
      acc += Tab::kM == 0 || g < 0 ? chunk_gather<float, ACC>(q + begin, dst, len, f)
                   : chunk_gather_strided<float, ACC>(q, tab.geom[g], begin, dst, len, small, f);
    } else if (dtype == EFCP_BF16) {
      const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p);
      acc += Tab::kM == 0 || g < 0 ? chunk_gather<__nv_bfloat16, ACC>(q + begin, dst, len, f)
                   : chunk_gather_strided<__nv_bfloat16, ACC>(q, tab.geom[g], begin, dst, len,
                                                              small, f);
    } else {
      const __half* q = static_cast<const __half*>(p);
      acc += Tab::kM == 0 || g < 0 ? chunk_gather<__half, ACC>(q + begin, dst, len, f)
                   : chunk_gather_strided<__half, ACC>(q, tab.geom[g], begin, dst, len, small, f);
    }
  }
  if (ACC) {
    if (finish_sum(acc, ws, first_launch) && norm) *norm = float(scale * sqrt(ws->sumsq));
  }
}

// The norm of a list without elements.
__global__ void k_grads_zero(Work* ws, float* norm) {
  ws->sumsq = 0.0;
  if (norm) *norm = 0.f;
}

// ------------------------------------------------------------------ host
struct Dim {
  long long size, stride;
};

// The layout of t with dimensions of size 1 dropped and neighbours merged, dims[0] running
// fastest in the flat vector.  Returns their number, or -1 when the descriptor is not valid.
int merge_dims(const efcp_tensor& t, Dim (&dims)[EFCP_MAX_RANK]) {
  if (t.rank == 0) {
    dims[0] = {t.numel, 1};
    return 1;
  }
  int n = 0;
  long long prod = 1;
  for (int k = t.rank - 1; k >= 0; --k) {
    const long long s = t.size[k], st = t.stride[k];
    if (s < 0 || st < 0) return -1;
    if (s > 1 && st > (1ll << 56) / s) return -1;  // beyond any address space
    if (s != 0 && prod > t.numel / s) return -1;  // the product would exceed numel
    prod *= s;
    if (s == 1) continue;
    if (n && st == dims[n - 1].size * dims[n - 1].stride) dims[n - 1].size *= s;
    else dims[n++] = {s, st};
  }
  if (prod != t.numel) return -1;
  if (!n) dims[n++] = {1, 1};
  if (n == 1 && dims[0].size == 1) dims[0].stride = 1;
  return n;
}

enum class Layout { kLinear, kDense, kStrided };

// kLinear: one after another in the flat order; kDense: the elements fill their memory, in
// another order; kStrided: anything else.  *overlaps: two elements may share memory.
Layout layout_of(const Dim* dims, int n, bool* overlaps) {
  *overlaps = false;
  if (n == 1 && dims[0].stride == 1) return Layout::kLinear;
  Dim by[EFCP_MAX_RANK];
  std::copy(dims, dims + n, by);
  std::sort(by, by + n, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  long long extent = 1;  // 1 + the largest position so far
  bool dense = true;
  for (int k = 0; k < n; ++k) {
    if (by[k].stride != extent) dense = false;
    if (by[k].stride < extent) *overlaps = true;
    extent += (by[k].size - 1) * by[k].stride;
  }
  return dense ? Layout::kDense : Layout::kStrided;
}

// Whether two tensors of a list share a byte.  Their positions in bytes are
//     a + sum i_k s_k  and  b + sum j_k t_k,   0 <= i_k < n_k, 0 <= j_k < m_k,
// and they share one where the difference of two positions lies between minus the width of an element of the
// one and the width of one of the other.  As a sum over all dimensions, largest stride first, every index is
// bounded by what the smaller strides can still make up for, which for slices of one tensor (columns of a
// matrix, channels of a kernel) leaves one or two values of it.  Layouts that need more than kShareSteps
// steps count as sharing.
class Sharing {
 public:
  struct Side {
    long long at;  // address
    int width, n;  // bytes of an element; dimensions
    const Dim* dim;
  };
  static bool any(const Side& a, const Side& b) {
    Sharing s;
    for (const Side* t : {&a, &b}) {
      for (int k = 0; k < t->n; ++k) {
        if (t->dim[k].size < 2) continue;
        const bool first = t == &a;
        s.term_[s.terms_++] = {t->dim[k].stride * t->width, first ? 0 : 1 - t->dim[k].size,
                               first ? t->dim[k].size - 1 : 0};
      }
    }
    std::sort(s.term_, s.term_ + s.terms_, [](const Term& x, const Term& y) { return x.step > y.step; });
    // equal strides are one term
    int n = 0;
    for (int k = 0; k < s.terms_; ++k) {
      if (n && s.term_[n - 1].step == s.term_[k].step) {
        s.term_[n - 1].lo += s.term_[k].lo;
        s.term_[n - 1].hi += s.term_[k].hi;
      } else {
        s.term_[n++] = s.term_[k];
      }
    }
    s.terms_ = n;
    for (int k = n; k-- > 0;) {
      s.low_[k] = s.low_[k + 1] + s.term_[k].step * s.term_[k].lo;
      s.high_[k] = s.high_[k + 1] + s.term_[k].step * s.term_[k].hi;
    }
    // position in a minus position in b: above -width of a, below width of b
    return s.reach(0, b.at - a.at - a.width + 1, b.at - a.at + b.width - 1);
  }

 private:
  struct Term {
    long long step, lo, hi;  // bytes; bounds of the index
  };
  static constexpr int kShareSteps = 4096;
  Term term_[2 * EFCP_MAX_RANK];
  long long low_[2 * EFCP_MAX_RANK + 1] = {}, high_[2 * EFCP_MAX_RANK + 1] = {};  // of the terms from k on
  int terms_ = 0, steps_ = 0;

  static long long floor_div(long long a, long long b) { return a / b - (a % b < 0); }
  // Whether the terms from k on can add up to something from lo to hi.
  bool reach(int k, long long lo, long long hi) {
    if (++steps_ > kShareSteps) return true;
    if (hi < low_[k] || lo > high_[k]) return false;
    if (k == terms_) return true;
    const Term& t = term_[k];
    if (t.step == 0) return reach(k + 1, lo, hi);
    const long long first = std::max(t.lo, -floor_div(high_[k + 1] - lo, t.step));
    const long long last = std::min(t.hi, floor_div(hi - low_[k + 1], t.step));
    for (long long i = first; i <= last; ++i)
      if (reach(k + 1, lo - i * t.step, hi - i * t.step)) return true;
    return false;
  }
};

enum class Op { kNorm, kClip, kGather };

// A tensor of the list that a launch has to deal with.
struct Entry {
  void* data;
  int64_t numel, dst;
  int dtype, dims;  // dims 0: no layout needed
  Dim dim[4];
};

// Checks the list and describes its tensors; `sum` receives the number of elements.  Empty tensors are
// left out, absent ones too unless the list is gathered.  A layout is noted where the elements lie
// neither one after another nor, if any order will do, close together.
int read_list(const efcp_tensor* grads, int n, Op op, std::vector<Entry>* out, int64_t* sum) {
  int64_t total = 0;
  if (n < 0 || (n && !grads)) return EFCP_EINVAL;
  out->reserve(size_t(n));
  for (int i = 0; i < n; ++i) {
    const efcp_tensor& t = grads[i];
    if (t.numel < 0 || t.numel > (1ll << 40) || t.rank < 0 || t.rank > EFCP_MAX_RANK ||
        t.dtype < 0 || t.dtype > 2)
      return EFCP_EINVAL;
    if (total > INT64_MAX / 8 - t.numel) return EFCP_EINVAL;
    Entry e{t.data, t.numel, total, t.dtype, 0, {}};
    total += t.numel;
    if (!t.numel) continue;
    if (!t.data) {
      if (op == Op::kGather) out->push_back(e);
      continue;
    }
    const uintptr_t size = t.dtype == EFCP_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(t.data) % size) return EFCP_EINVAL;
    if (t.rank) {
      Dim dims[EFCP_MAX_RANK];
      bool overlaps = false;
      const int nd = merge_dims(t, dims);
      if (nd < 0) return EFCP_EINVAL;
      const Layout l = layout_of(dims, nd, &overlaps);
      if (overlaps && op == Op::kClip) return EFCP_EINVAL;
      if (l == Layout::kStrided || (l == Layout::kDense && op == Op::kGather)) {
        if (nd > 4) return EFCP_EINVAL;
        e.dims = nd;
        std::copy(dims, dims + nd, e.dim);
      }
    }
    out->push_back(e);
  }
  *sum = total;
  return EFCP_OK;
}

// Whether two of the tensors share memory.
bool list_overlaps(const efcp_tensor* grads, int n) {
  struct Range {
    long long begin, end;  // addresses
    int index;
  };
  std::vector<Range> r;
  r.reserve(size_t(n));
  const auto side = [&](int i, Dim (&dims)[EFCP_MAX_RANK]) {
    const efcp_tensor& t = grads[i];
    const int nd = merge_dims(t, dims);
    return Sharing::Side{static_cast<long long>(reinterpret_cast<intptr_t>(t.data)),
                         t.dtype == EFCP_F32 ? 4 : 2, nd, dims};
  };
  bool sorted = true;
  long long reached = 0;
  for (int i = 0; i < n; ++i) {
    if (!grads[i].numel || !grads[i].data) continue;
    Dim dims[EFCP_MAX_RANK];
    const Sharing::Side s = side(i, dims);
    long long last = 0;
    for (int k = 0; k < s.n; ++k) last += (dims[k].size - 1) * dims[k].stride;
    const Range q{s.at, s.at + (last + 1) * s.width, i};
    sorted = sorted && q.begin >= reached;
    reached = q.end;
    r.push_back(q);
  }
  if (sorted) return false;
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  // ranges that begin inside an earlier one: that pair has to be looked at
  std::vector<const Range*> open;
  for (const Range& q : r) {
    open.erase(std::remove_if(open.begin(), open.end(),
                              [&](const Range* o) { return o->end <= q.begin; }),
               open.end());
    for (const Range* o : open) {
      Dim a[EFCP_MAX_RANK], b[EFCP_MAX_RANK];
      if (Sharing::any(side(o->index, a), side(q.index, b))) return true;
    }
    open.push_back(&q);
  }
  return false;
}

// n / d = n * mul >> shift for n < 2^31: with 2^b >= d, mul = floor(2^(31 + b) / d) + 1 is off from
// 2^(31 + b) / d by at most 1, so the quotient by less than n / 2^(31 + b) < 1 / d.
void set_divisor(long long d, unsigned* mul, unsigned char* shift) {
  if (d >= (1ll << 31)) d = (1ll << 31) - 1;  // (not used: such a tensor takes 64-bit divisions)
  int b = 0;
  while ((1ll << b) < d) ++b;
  *shift = static_cast<unsigned char>(31 + b);
  *mul = unsigned(((1ull << (31 + b)) / static_cast<unsigned long long>(d)) + 1);
}

// Fills the table from list[*at] on, until it is full or the list ends.  Chunk numbers are 32-bit: a
// tensor has at most 2^28 chunks of 32 KB (only short lists have smaller ones), and no
// tensor is added to 2^30 of them.
template <class Tab>
void fill(Tab& tab, const std::vector<Entry>& list, int chunk_log, size_t* at) {
  tab.chunk_log = chunk_log;
  int used = 0, shapes = 0;
  unsigned chunks = 0;
  for (; *at < list.size() && used < Tab::kN && chunks < (1u << 30); ++*at, ++used) {
    const Entry& e = list[*at];
    int shape = -1;
    if (Tab::kM > 0 && e.dims) {
      if (shapes == Tab::kM) break;
      shape = shapes++;
      Geom& g = tab.geom[shape];
      for (int k = 0; k < 3; ++k) g.size[k] = k < e.dims ? e.dim[k].size : 1;
      for (int k = 0; k < 4; ++k) g.stride[k] = k < e.dims ? e.dim[k].stride : 0;
      for (int k = 0; k < 3; ++k) set_divisor(g.size[k], &g.mul[k], &g.shift[k]);
    }
    const int64_t per = 1ll << (chunk_log - (e.dtype == EFCP_F32 ? 2 : 1));
    tab.ptr[used] = e.data;
    tab.numel[used] = e.numel;
    tab.dst[used] = e.dst;
    tab.first[used] = chunks;
    tab.shape[used] = short(shape);
    tab.dtype[used] = static_cast<unsigned char>(e.dtype);
    chunks += unsigned((e.numel + per - 1) / per);
  }
  tab.n = used;
  tab.first[used] = chunks;
}

struct Args {
  const std::vector<Entry>& list;
  float* flat;
  double max_norm, scale;
  float* norm;
  Work* ws;
  cudaStream_t st;
  int sms, chunk_log;
};

// The largest chunks that still give every SM eight of them (301 ragged fp16 tensors of 42 MB: 42 us, with four
// 44, with sixteen 46; then the way to a chunk's tensor costs more than the even shares save).
int pick_chunk_log(const std::vector<Entry>& list, int sms) {
  int64_t bytes = 0;
  for (const Entry& e : list)
    if (e.data) bytes += e.numel * (e.dtype == EFCP_F32 ? 4 : 2);
  int log = kGrChunkLog;
  while (log > kGrChunkLogMin && (bytes >> log) < 8ll * sms) --log;
  return log;
}

enum class Kernel { kSumsq, kScale, kGather, kGatherClip, kGatherNorm };

// One pass over the list: a launch for as many tensors at a time as a table holds.
template <class Tab>
int run_pass(const Args& a, Kernel kern) {
  Tab tab;
  size_t at = 0;
  bool first = true;
  while (at < a.list.size()) {
    fill(tab, a.list, a.chunk_log, &at);
    const unsigned chunks = tab.first[tab.n];
    const Shape shape{
        std::min<unsigned>(chunks, unsigned(std::min(a.sms * kGrBlocksPerSM, kGrMaxBlocks))),
        kGrThreads, 0, 0};
    cudaError_t e = cudaSuccess;
    switch (kern) {
      case Kernel::kSumsq:
        e = launch(k_grads_sumsq<Tab>, shape, a.st, tab, a.ws, first, a.scale, a.norm);
        break;
      case Kernel::kScale:
        e = launch(k_grads_scale<Tab>, shape, a.st, tab, static_cast<const Work*>(a.ws), a.max_norm,
                   a.scale);
        break;
      case Kernel::kGather:
        e = launch(k_grads_gather<Tab, false, false>, shape, a.st, tab, a.flat, a.ws, first, a.max_norm,
                   a.scale, a.norm);
        break;
      case Kernel::kGatherClip:
        e = launch(k_grads_gather<Tab, true, false>, shape, a.st, tab, a.flat, a.ws, first, a.max_norm,
                   a.scale, a.norm);
        break;
      case Kernel::kGatherNorm:
        e = launch(k_grads_gather<Tab, false, true>, shape, a.st, tab, a.flat, a.ws, first, a.max_norm,
                   a.scale, a.norm);
        break;
    }
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      return EFCP_ECUDA;
    }
    first = false;
  }
  if (first && (kern == Kernel::kSumsq || kern == Kernel::kGatherNorm)) {
    k_grads_zero<<<1, 1, 0, a.st>>>(a.ws, a.norm);
    if (cudaGetLastError() != cudaSuccess) return EFCP_ECUDA;
  }
  return EFCP_OK;
}

// The table's size follows the list's: parameters are copied with every launch.
using LargeTable = Table<600, 150>;
using LargeDenseTable = Table<960, 0>;
static_assert(sizeof(LargeTable) + 64 <= 32764 && sizeof(LargeDenseTable) + 64 <= 32764,
              "kernel parameters");

int run_pass_sized(const Args& a, Kernel kern) {
  size_t shapes = 0;
  const size_t n = a.list.size();
  for (const Entry& e : a.list) shapes += e.dims > 0;
  if (!shapes) {
    if (n <= 96) return run_pass<Table<96, 0>>(a, kern);
    if (n <= 320) return run_pass<Table<320, 0>>(a, kern);
    return run_pass<LargeDenseTable>(a, kern);
  }
  if (n <= 96 && shapes <= 32) return run_pass<Table<96, 32>>(a, kern);
  return run_pass<LargeTable>(a, kern);
}

// The host side keeps the list in a vector: running out of memory is an error code, not an exception.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (...) {
    return EFCP_ENOMEM;
  }
}

bool bad_scalar(float v) { return !(v > 0.f) || !std::isfinite(v); }

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

int64_t efcp_grads_workspace_bytes(void) { return int64_t(sizeof(Work)); }

int efcp_grads_norm(const efcp_tensor* grads, int32_t n, float scale, float* norm,
                    void* workspace, void* stream) {
  if (!norm || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 7) || bad_scalar(scale))
    return EFCP_EINVAL;
  return guarded([&] {
    std::vector<Entry> list;
    int64_t sum = 0;
    const int rc = read_list(grads, n, Op::kNorm, &list, &sum);
    if (rc != EFCP_OK) return rc;
    Args a{list, nullptr, 0.0, double(scale), norm, static_cast<Work*>(workspace),
           static_cast<cudaStream_t>(stream), device_sms(), 0};
    if (a.sms < 1) return EFCP_ECUDA;
    a.chunk_log = pick_chunk_log(list, a.sms);
    return run_pass_sized(a, Kernel::kSumsq);
  });
}

int efcp_grads_clip(const efcp_tensor* grads, int32_t n, float max_norm, float scale, float* norm,
                    void* workspace, void* stream) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7) || bad_scalar(scale) ||
      !(max_norm > 0.f))
    return EFCP_EINVAL;
  return guarded([&] {
    std::vector<Entry> list;
    int64_t sum = 0;
    int rc = read_list(grads, n, Op::kClip, &list, &sum);
    if (rc != EFCP_OK) return rc;
    if (list_overlaps(grads, n)) return EFCP_EINVAL;
    Args a{list, nullptr, double(max_norm), double(scale), norm, static_cast<Work*>(workspace),
           static_cast<cudaStream_t>(stream), device_sms(), 0};
    if (a.sms < 1) return EFCP_ECUDA;
    a.chunk_log = pick_chunk_log(list, a.sms);
    rc = run_pass_sized(a, Kernel::kSumsq);
    return rc != EFCP_OK ? rc : run_pass_sized(a, Kernel::kScale);
  });
}

int efcp_grads_gather(const efcp_tensor* grads, int32_t n, float* flat, int64_t d, float max_norm,
                      float scale, float* norm, void* workspace, void* stream) {
  if ((!flat && d != 0) || (reinterpret_cast<uintptr_t>(flat) & 3) || bad_scalar(scale) ||
      !(max_norm >= 0.f))
    return EFCP_EINVAL;
  if ((max_norm > 0.f || norm) &&
      (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)))
    return EFCP_EINVAL;
  return guarded([&] {
    std::vector<Entry> list, unordered;
    int64_t sum = 0;
    int rc = read_list(grads, n, Op::kGather, &list, &sum);
    if (rc != EFCP_OK) return rc;
    if (sum != d) return EFCP_EINVAL;
    Args a{list, flat, double(max_norm), double(scale), norm, static_cast<Work*>(workspace),
           static_cast<cudaStream_t>(stream), device_sms(), 0};
    if (a.sms < 1) return EFCP_ECUDA;
    a.chunk_log = pick_chunk_log(list, a.sms);
    if (max_norm == 0.f) return run_pass_sized(a, norm ? Kernel::kGatherNorm : Kernel::kGather);
    rc = read_list(grads, n, Op::kNorm, &unordered, &sum);  // most layouts do not matter to the norm
    if (rc != EFCP_OK) return rc;
    Args b{unordered, nullptr, 0.0, a.scale, norm, a.ws, a.st, a.sms, a.chunk_log};
    rc = run_pass_sized(b, Kernel::kSumsq);
    return rc != EFCP_OK ? rc : run_pass_sized(a, Kernel::kGatherClip);
  });
}

}  // extern "C"
