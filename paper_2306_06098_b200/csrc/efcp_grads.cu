// The gradients of a model as a list of tensors: global norm, clipping, and the gather into the
// flat fp32 vector that the optimizer step reads (see include/efcp.h).
//
// All three are streams over memory with a handful of operations per element: HBM bounds them when
// the list is large, the launch when it is small.  The list travels in the kernel's parameters (up to
// 32 KB of constant memory: no copy to wait for, no host buffer that has to outlive the
// call).  It is cut into chunks of 16 KB that the thread blocks take in turn, so that one
// large matrix and hundreds of short vectors both keep every SM busy.
#include "efcp.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "efcp_common.cuh"
#include "efcp_device.h"
#include "efcp_num.cuh"

namespace efcp {
namespace {

constexpr int kGrThreads = 256;
constexpr int kGrBlocksPerSM = 8;
constexpr int kGrMaxBlocks = 4096;    // partial sums the workspace has room for
constexpr int kGrChunkBytes = 16384;  // of the source; 64 bytes per thread

// A tensor's layout when its elements do not lie one after another: up to four merged
// dimensions, [0] running fastest in the flat vector.
struct Geom {
  long long size[3];  // of dimensions 0..2 (dimension 3 is what is left)
  long long stride[4];
};

// What a launch works on.  first[i] is the number of the first chunk of tensor i.
template <int N, int M>
struct Table {
  static constexpr int kN = N, kM = M;
  const void* ptr[N];
  long long numel[N];
  long long dst[N];  // position in the flat vector
  Geom geom[M];
  unsigned first[N + 1];
  int n;
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
__device__ __forceinline__ int chunk_elems(int dtype) {
  return dtype == EFCP_F32 ? kGrChunkBytes / 4 : kGrChunkBytes / 2;
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
  if (small) {  // fewer than 2^31 elements: 32-bit divisions
    unsigned r = unsigned(e);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const unsigned s = unsigned(g.size[k]), q = r / s;
      pos += (long long)(r - q * s) * g.stride[k];
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

// Sum of the squares of V values.  fp32 products and sums are exact to a few 2^-24 as long as
// they neither overflow nor vanish; otherwise the same values are squared in fp64.
template <int V>
__device__ __forceinline__ double sumsq_of(const float (&v)[V]) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) s = fmaf(v[j], v[j], s);
  if (s > 1e-28f && s < 1e37f) return double(s);
  double t = 0.0;
#pragma unroll
  for (int j = 0; j < V; ++j) t = fma(double(v[j]), double(v[j]), t);
  return t;
}

template <typename T>
__device__ __forceinline__ double chunk_sumsq(const T* p, int len) {
  constexpr int V = 16 / int(sizeof(T));
  using P = Pack<T, V>;
  // elements before the first 16-byte boundary
  const int skew = int((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
  const int head = min(len, skew ? V - skew : 0);
  const int nv = (len - head) / V;
  const P* q = reinterpret_cast<const P*>(p + head);
  double acc = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += kGrThreads) {
    const P a = q[i];
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = to_f32(a.v[j]);
    acc += sumsq_of(v);
  }
  const int rest = len - head - nv * V;  // the ends: fewer than 2 V elements
  if (int(threadIdx.x) < head + rest) {
    const int i = int(threadIdx.x) < head ? int(threadIdx.x) : nv * V + int(threadIdx.x);
    const double x = double(to_f32(p[i]));
    acc += x * x;
  }
  return acc;
}

template <typename T>
__device__ double chunk_sumsq_strided(const T* p, const Geom& g, long long begin, int len,
                                      bool small) {
  double acc = 0.0;
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
__global__ void __launch_bounds__(kGrThreads)
    k_grads_sumsq(const __grid_constant__ Tab tab, Work* ws, bool first_launch, double scale,
                  float* norm) {
  double acc = 0.0;
  const unsigned total = tab.first[tab.n];
  for (unsigned c = blockIdx.x; c < total; c += gridDim.x) {
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = tab.shape[i];
    if (g < 0) {
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
__global__ void __launch_bounds__(kGrThreads)
    k_grads_scale(const __grid_constant__ Tab tab, const Work* ws, double max_norm, double scale) {
  const float f = factor_of(ws, max_norm, scale);
  if (f == 1.f) return;
  const unsigned total = tab.first[tab.n];
  for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
    const unsigned c = total - 1 - b;
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = tab.shape[i];
    void* p = const_cast<void*>(tab.ptr[i]);
    const bool small = tab.numel[i] < (1ll << 31);
    if (dtype == EFCP_F32) {
      if (g < 0) chunk_scale(static_cast<float*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<float*>(p), tab.geom[g], begin, len, small, f);
    } else if (dtype == EFCP_BF16) {
      if (g < 0) chunk_scale(static_cast<__nv_bfloat16*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<__nv_bfloat16*>(p), tab.geom[g], begin, len, small, f);
    } else {
      if (g < 0) chunk_scale(static_cast<__half*>(p) + begin, len, f);
      else chunk_scale_strided(static_cast<__half*>(p), tab.geom[g], begin, len, small, f);
    }
  }
}

// v f, or v itself when f is 1: the select is on the bits, so that a copy keeps every bit of a NaN.
__device__ __forceinline__ float scaled(float v, float f) {
  return __uint_as_float(f == 1.f ? __float_as_uint(v) : __float_as_uint(__fmul_rn(v, f)));
}

// One chunk into the flat vector; with ACC its sum of squares is returned.  Four elements per
// access: the stores are then 16 bytes from consecutive lanes whatever the source's type.
template <typename T, bool ACC>
__device__ __forceinline__ double chunk_gather(const T* p, float* dst, int len, float f) {
  using P = Pack<T, 4>;
  double acc = 0.0;
  int done = 0;
  if (!(reinterpret_cast<uintptr_t>(p) & (sizeof(P) - 1)) &&
      !(reinterpret_cast<uintptr_t>(dst) & 15)) {
    const P* q = reinterpret_cast<const P*>(p);
    float4* o = reinterpret_cast<float4*>(dst);
    const int nv = len / 4;
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += kGrThreads) {
      const P a = q[i];
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = to_f32(a.v[j]);
      if (ACC) acc += sumsq_of(v);
      o[i] = make_float4(scaled(v[0], f), scaled(v[1], f), scaled(v[2], f), scaled(v[3], f));
    }
    done = nv * 4;
  }
#pragma unroll 4
  for (int i = done + threadIdx.x; i < len; i += kGrThreads) {
    const float v = to_f32(p[i]);
    if (ACC) acc += double(v) * double(v);
    dst[i] = scaled(v, f);
  }
  return acc;
}

template <typename T, bool ACC>
__device__ double chunk_gather_strided(const T* p, const Geom& g, long long begin, float* dst,
                                       int len, bool small, float f) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < len; i += kGrThreads) {
    const float v = to_f32(p[strided_pos(g, begin + i, small)]);
    if (ACC) acc += double(v) * double(v);
    dst[i] = scaled(v, f);
  }
  return acc;
}

// CLIP: the factor comes from the norm a launch before has left in ws.  ACC: there is no
// clipping, and the norm is taken in the same pass.
template <class Tab, bool CLIP, bool ACC>
__global__ void __launch_bounds__(kGrThreads)
    k_grads_gather(const __grid_constant__ Tab tab, float* flat, Work* ws, bool first_launch,
                   double max_norm, double scale, float* norm) {
  const float f = CLIP ? factor_of(ws, max_norm, scale) : float(scale);
  const unsigned total = tab.first[tab.n];
  double acc = 0.0;
  for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
    const unsigned c = CLIP ? total - 1 - b : b;  // backwards after a norm, as k_grads_scale
    const int i = find_tensor(tab, c);
    const int dtype = tab.dtype[i], per = chunk_elems(dtype);
    const long long begin = (long long)(c - tab.first[i]) * per;
    const int len = int(min((long long)per, tab.numel[i] - begin));
    const int g = tab.shape[i];
    const void* p = tab.ptr[i];
    float* dst = flat + tab.dst[i] + begin;
    const bool small = tab.numel[i] < (1ll << 31);
    if (!p) {
      for (int j = threadIdx.x; j < len; j += kGrThreads) dst[j] = 0.f;
    } else if (dtype == EFCP_F32) {
      const float* q = static_cast<const float*>(p);
      acc += g < 0 ? chunk_gather<float, ACC>(q + begin, dst, len, f)
                   : chunk_gather_strided<float, ACC>(q, tab.geom[g], begin, dst, len, small, f);
    } else if (dtype == EFCP_BF16) {
      const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p);
      acc += g < 0 ? chunk_gather<__nv_bfloat16, ACC>(q + begin, dst, len, f)
                   : chunk_gather_strided<__nv_bfloat16, ACC>(q, tab.geom[g], begin, dst, len,
                                                              small, f);
    } else {
      const __half* q = static_cast<const __half*>(p);
      acc += g < 0 ? chunk_gather<__half, ACC>(q + begin, dst, len, f)
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

enum class Op { kNorm, kClip, kGather };

int check_list(const efcp_tensor* grads, int n, Op op, int64_t* sum) {
  int64_t total = 0;
  if (n < 0 || (n && !grads)) return EFCP_EINVAL;
  for (int i = 0; i < n; ++i) {
    const efcp_tensor& t = grads[i];
    if (t.numel < 0 || t.numel > (1ll << 40) || t.rank < 0 || t.rank > EFCP_MAX_RANK || t.dtype < 0 || t.dtype > 2)
      return EFCP_EINVAL;
    if (total > INT64_MAX / 8 - t.numel) return EFCP_EINVAL;
    total += t.numel;
    if (!t.numel || !t.data) continue;
    const uintptr_t size = t.dtype == EFCP_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(t.data) % size) return EFCP_EINVAL;
    if (t.rank) {
      Dim dims[EFCP_MAX_RANK];
      bool overlaps = false;
      const int nd = merge_dims(t, dims);
      if (nd < 0) return EFCP_EINVAL;
      const Layout l = layout_of(dims, nd, &overlaps);
      if (overlaps && op == Op::kClip) return EFCP_EINVAL;
      if (nd > 4 && (l == Layout::kStrided || op == Op::kGather)) return EFCP_EINVAL;
    }
  }
  *sum = total;
  return EFCP_OK;
}

// Fills the table from grads[*at] on, until it is full or the list ends.  Chunk numbers are
// 32-bit: a tensor has at most 2^28 chunks, and no tensor is added to 2^30 of them.
template <class Tab>
void fill(Tab& tab, const efcp_tensor* grads, int n, Op op, int* at, int64_t* dst) {
  int used = 0, shapes = 0;
  unsigned chunks = 0;
  for (; *at < n && used < Tab::kN && shapes < Tab::kM && chunks < (1u << 30); ++*at) {
    const efcp_tensor& t = grads[*at];
    const int64_t here = *dst;
    *dst += t.numel;
    if (!t.numel || (!t.data && op != Op::kGather)) continue;
    int shape = -1;
    if (t.rank && t.data) {
      Dim dims[EFCP_MAX_RANK];
      bool overlaps;
      const int nd = merge_dims(t, dims);
      const Layout l = layout_of(dims, nd, &overlaps);
      if (l == Layout::kStrided || (l == Layout::kDense && op == Op::kGather)) {
        shape = shapes++;
        Geom& g = tab.geom[shape];
        for (int k = 0; k < 3; ++k) g.size[k] = k < nd ? dims[k].size : 1;
        for (int k = 0; k < 4; ++k) g.stride[k] = k < nd ? dims[k].stride : 0;
      }
    }
    const int64_t per = kGrChunkBytes / (t.dtype == EFCP_F32 ? 4 : 2);
    tab.ptr[used] = t.data;
    tab.numel[used] = t.numel;
    tab.dst[used] = here;
    tab.first[used] = chunks;
    tab.shape[used] = short(shape);
    tab.dtype[used] = static_cast<unsigned char>(t.dtype);
    chunks += unsigned((t.numel + per - 1) / per);
    ++used;
  }
  tab.n = used;
  tab.first[used] = chunks;
}

struct Args {
  const efcp_tensor* grads;
  int n;
  float* flat;
  double max_norm, scale;
  float* norm;
  Work* ws;
  cudaStream_t st;
  int sms;
};

enum class Kernel { kSumsq, kScale, kGather, kGatherClip, kGatherNorm };

// One pass over the list: a launch for as many tensors at a time as a table holds.
template <class Tab>
int run_pass(const Args& a, Op op, Kernel kern) {
  Tab tab;
  int at = 0;
  int64_t dst = 0;
  bool first = true;
  while (at < a.n) {
    fill(tab, a.grads, a.n, op, &at, &dst);
    const unsigned chunks = tab.first[tab.n];
    if (!chunks) continue;
    const unsigned grid = std::min<unsigned>(
        chunks, unsigned(std::min(a.sms * kGrBlocksPerSM, kGrMaxBlocks)));
    switch (kern) {
      case Kernel::kSumsq:
        k_grads_sumsq<<<grid, kGrThreads, 0, a.st>>>(tab, a.ws, first, a.scale, a.norm);
        break;
      case Kernel::kScale:
        k_grads_scale<<<grid, kGrThreads, 0, a.st>>>(tab, a.ws, a.max_norm, a.scale);
        break;
      case Kernel::kGather:
        k_grads_gather<Tab, false, false><<<grid, kGrThreads, 0, a.st>>>(
            tab, a.flat, a.ws, first, a.max_norm, a.scale, a.norm);
        break;
      case Kernel::kGatherClip:
        k_grads_gather<Tab, true, false><<<grid, kGrThreads, 0, a.st>>>(
            tab, a.flat, a.ws, first, a.max_norm, a.scale, a.norm);
        break;
      case Kernel::kGatherNorm:
        k_grads_gather<Tab, false, true><<<grid, kGrThreads, 0, a.st>>>(
            tab, a.flat, a.ws, first, a.max_norm, a.scale, a.norm);
        break;
    }
    if (cudaGetLastError() != cudaSuccess) return EFCP_ECUDA;
    first = false;
  }
  if (first && (kern == Kernel::kSumsq || kern == Kernel::kGatherNorm)) {
    k_grads_zero<<<1, 1, 0, a.st>>>(a.ws, a.norm);
    if (cudaGetLastError() != cudaSuccess) return EFCP_ECUDA;
  }
  return EFCP_OK;
}

// The table's size follows the list's: parameters are copied with every launch.
using SmallTable = Table<64, 24>;
using MidTable = Table<320, 96>;
using LargeTable = Table<600, 200>;
static_assert(sizeof(LargeTable) + 64 <= 32764, "kernel parameters");

int run_pass_sized(const Args& a, Op op, Kernel kern) {
  int shapes = 0;
  for (int i = 0; i < a.n; ++i) shapes += a.grads[i].rank > 0;
  if (a.n <= SmallTable::kN && shapes <= SmallTable::kM) return run_pass<SmallTable>(a, op, kern);
  if (a.n <= MidTable::kN && shapes <= MidTable::kM) return run_pass<MidTable>(a, op, kern);
  return run_pass<LargeTable>(a, op, kern);
}

bool bad_scalar(float v) { return !(v > 0.f) || !std::isfinite(v); }

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

int64_t efcp_grads_workspace_bytes(void) { return int64_t(sizeof(Work)); }

int efcp_grads_norm(const efcp_tensor* grads, int32_t n, float scale, float* norm,
                    void* workspace, void* stream) {
  int64_t d = 0;
  if (!norm || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 7) || bad_scalar(scale))
    return EFCP_EINVAL;
  const int rc = check_list(grads, n, Op::kNorm, &d);
  if (rc != EFCP_OK) return rc;
  Args a{grads, n, nullptr, 0.0, double(scale), norm, static_cast<Work*>(workspace),
         static_cast<cudaStream_t>(stream), device_sms()};
  if (a.sms < 1) return EFCP_ECUDA;
  return run_pass_sized(a, Op::kNorm, Kernel::kSumsq);
}

int efcp_grads_clip(const efcp_tensor* grads, int32_t n, float max_norm, float scale, float* norm,
                    void* workspace, void* stream) {
  int64_t d = 0;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7) || bad_scalar(scale) ||
      !(max_norm > 0.f))
    return EFCP_EINVAL;
  int rc = check_list(grads, n, Op::kClip, &d);
  if (rc != EFCP_OK) return rc;
  Args a{grads, n, nullptr, double(max_norm), double(scale), norm,
         static_cast<Work*>(workspace), static_cast<cudaStream_t>(stream), device_sms()};
  if (a.sms < 1) return EFCP_ECUDA;
  rc = run_pass_sized(a, Op::kNorm, Kernel::kSumsq);
  return rc != EFCP_OK ? rc : run_pass_sized(a, Op::kClip, Kernel::kScale);
}

int efcp_grads_gather(const efcp_tensor* grads, int32_t n, float* flat, int64_t d, float max_norm,
                      float scale, float* norm, void* workspace, void* stream) {
  int64_t sum = 0;
  if ((!flat && d != 0) || (reinterpret_cast<uintptr_t>(flat) & 3) || bad_scalar(scale) ||
      !(max_norm >= 0.f))
    return EFCP_EINVAL;
  if ((max_norm > 0.f || norm) &&
      (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)))
    return EFCP_EINVAL;
  int rc = check_list(grads, n, Op::kGather, &sum);
  if (rc != EFCP_OK) return rc;
  if (sum != d) return EFCP_EINVAL;
  Args a{grads, n, flat, double(max_norm), double(scale), norm, static_cast<Work*>(workspace),
         static_cast<cudaStream_t>(stream), device_sms()};
  if (a.sms < 1) return EFCP_ECUDA;
  if (max_norm > 0.f) {
    rc = run_pass_sized(a, Op::kNorm, Kernel::kSumsq);
    return rc != EFCP_OK ? rc : run_pass_sized(a, Op::kGather, Kernel::kGatherClip);
  }
  return run_pass_sized(a, Op::kGather, norm ? Kernel::kGatherNorm : Kernel::kGather);
}

}  // extern "C"
