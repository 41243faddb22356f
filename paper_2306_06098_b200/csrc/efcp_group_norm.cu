// Group normalisation with an activation on channels-last tensors, forward and backward (the
// formulas stand in include/efcp.h).
//
// Memory bounds it: forward x is read and y written once, backward x and dy are read and
// dx is written once, with 10 to 30 operations per element in between.
//
// A work item is one sample, a chunk of its rows and a tile of its channels; a tile is a number of
// whole groups.  A thread owns V neighbouring channels (one access of up to 16 bytes) and walks down
// the rows of the chunk, so the channel's weight, bias and statistics stay in its registers, and
// sums over rows stay in registers too until the block joins them.  Two passes over the input: the
// sums of all chunks, then the result.
#include "efcp.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "efcp_device.h"
#include "efcp_num.cuh"

namespace efcp {
namespace {

constexpr int kGnThreads = 256;
constexpr int kGnBlocksPerSM = 8;
constexpr int kGnMaxRowsPerThread = 64;
constexpr int kGnUnroll = 4;

struct Gn {
  const void* x;
  const void* dy;
  void* y;  // backward: dx
  const void* weight;
  const void* bias;
  float* mean;
  float* rstd;
  float* part;
  long long x_batch, x_row, y_batch, y_row, dy_batch, dy_row;
  long long rows, chunk_rows;  // rows of a sample, of a chunk
  int channels, groups, per;   // per: channels of a group
  int tile_groups, tiles;      // groups of a tile (the last tile may have fewer), tiles
  int chunks;                  // chunks of a sample
  int param_dtype;
  float eps;
};

// What a thread block works on.
struct Item {
  long long n, r0, r1;
  int chunk, g0, ng, c0, width;  // groups g0 .. g0 + ng, channels c0 .. c0 + width
  int cols;                      // vectors of a row handled side by side
  int lanes_rows;                // rows handled side by side
  int tx, ty;                    // this thread's place among them; ty >= lanes_rows: idle
};

template <int V>
__device__ __forceinline__ Item item_of(const Gn& p, unsigned b) {
  Item it;
  it.chunk = int(b % unsigned(p.chunks));
  b /= unsigned(p.chunks);
  const int tile = int(b % unsigned(p.tiles));
  it.n = b / unsigned(p.tiles);
  it.r0 = it.chunk * p.chunk_rows;
  it.r1 = min(p.rows, it.r0 + p.chunk_rows);
  it.g0 = tile * p.tile_groups;
  it.ng = min(p.tile_groups, p.groups - it.g0);
  it.c0 = it.g0 * p.per;
  it.width = it.ng * p.per;
  it.cols = min(it.width / V, kGnThreads);
  it.lanes_rows = kGnThreads / it.cols;
  it.tx = int(threadIdx.x) % it.cols;
  it.ty = int(threadIdx.x) / it.cols;
  return it;
}

// V elements as fp32, through the read-only path (the input is not written during the launch, so
// loads may move ahead of the stores of earlier rows).
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  Pack<T, V> a;
  if constexpr (sizeof(a) == 16) {
    *reinterpret_cast<uint4*>(&a) = __ldg(reinterpret_cast<const uint4*>(p));
  } else if constexpr (sizeof(a) == 4) {
    *reinterpret_cast<unsigned*>(&a) = __ldg(reinterpret_cast<const unsigned*>(p));
  } else {
    static_assert(sizeof(a) == 2, "2, 4 or 16 bytes");
    *reinterpret_cast<unsigned short*>(&a) = __ldg(reinterpret_cast<const unsigned short*>(p));
  }
  return a;
}
template <typename T, int V>
__device__ __forceinline__ void unpack(const Pack<T, V>& a, float (&v)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = to_f32(a.v[j]);
}

// Sum over groups of neighbouring lanes (a power of two of them), the same in all of them.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Lanes that join to reduce one group when the block has ng of them to reduce: 32 at most, and
// no more than keep the block's threads busy.
__device__ __forceinline__ int lanes_per_group(int ng) {
  int l = 32;
  while (l > 1 && l * ng > kGnThreads) l >>= 1;
  return l;
}

// act(z) and act'(z)
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
  if (ACT == EFCP_ACT_RELU) return z < 0.f ? 0.f : z;  // (a NaN stays one)
  if (ACT == EFCP_ACT_SILU) return z / (1.f + __expf(-z));
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_grad(float z) {
  if (ACT == EFCP_ACT_RELU) return z <= 0.f ? 0.f : 1.f;
  if (ACT == EFCP_ACT_SILU) {
    const float s = 1.f / (1.f + __expf(-z));
    return s * fmaf(z, 1.f - s, 1.f);
  }
  return 1.f;
}

// ------------------------------------------------------------------ forward
// Mean and sum of squared deviations of every group over a chunk of rows.
//
// A thread sums x - K and (x - K)^2 with K the first value it sees of a channel.  K is one of
// the values summed, so (K - mean)^2 is at most their sum of squared deviations, and what
// the subtraction of n (mean - K)^2 loses stays below n 2^-24 of the result, n <= 64 rows,
// whatever the mean of the data.  Threads, and then chunks, are joined by
//     mean = sum n_i mean_i / sum n_i,   M2 = sum M2_i + n_i (mean_i - mean)^2,
// two plain sums without cancellation.  The means are kept as differences from one value of
// the group, its first: a mean far from zero would otherwise round away what the
// second sum needs.
template <typename T, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_stats(const Gn p) {
  __shared__ float val[kGnThreads * V];
  __shared__ float cnt[kGnThreads];
  const Item it = item_of<V>(p, blockIdx.x);
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  // (row 0 of the sample, also for later chunks)
  float k[V], s1[V], s2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) k[j] = s1[j] = s2[j] = 0.f;
  int n = 0;
  if (it.ty < it.lanes_rows) {
    for (int col = it.tx; col < it.width / V; col += it.cols) {
      for (long long r = it.r0 + it.ty; r < it.r1; r += kGnUnroll * it.lanes_rows) {
        Pack<T, V> a[kGnUnroll];
#pragma unroll
        for (int u = 0; u < kGnUnroll; ++u) {
          const long long rr = r + (long long)u * it.lanes_rows;
          if (rr < it.r1) a[u] = load_pack<T, V>(x + rr * p.x_row + (long long)col * V);
        }
#pragma unroll
        for (int u = 0; u < kGnUnroll; ++u) {
          if (r + (long long)u * it.lanes_rows >= it.r1) break;
          float v[V];
          unpack(a[u], v);
          if (!n) {
#pragma unroll
            for (int j = 0; j < V; ++j) k[j] = v[j];
          }
          ++n;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float d = v[j] - k[j];
            s1[j] += d;
            s2[j] = fmaf(d, d, s2[j]);
          }
        }
      }
    }
  }
  // this thread's mean and M2 per channel
  const float inv = n ? 1.f / float(n) : 0.f;
  const int used = it.cols * V;  // values of a row in val
  const int per = min(p.per, used);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float m = s1[j] * inv;
    s2[j] = fmaxf(0.f, fmaf(-m, s1[j], s2[j]));
    const int g = (it.tx * V + j) / per;  // 0 when a group is wider than the block
    k[j] = n ? (k[j] - to_f32(x[(long long)g * p.per])) + m : 0.f;
    val[threadIdx.x * V + j] = k[j];
  }
  cnt[threadIdx.x] = float(n);
  __syncthreads();
  // groups: `lanes` neighbouring lanes each; a group's values lie in a row of `per` for each
  // of the rows handled side by side
  const int lanes = lanes_per_group(it.ng);
  const int items = per * it.lanes_rows;
  const float total = float(it.r1 - it.r0) * float(p.per);
  const int lane = int(threadIdx.x) % lanes, step = kGnThreads / lanes;
  float* part = p.part + ((it.n * p.chunks + it.chunk) * p.groups + it.g0) * 2;
  // every thread takes part in every round: the shuffles need whole warps
  for (int g0 = 0; g0 < it.ng; g0 += step) {
    const int g = g0 + int(threadIdx.x) / lanes;
    float s = 0.f;
    if (g < it.ng) {
      for (int i = lane; i < items; i += lanes) {
        const int at = (i / per) * used + g * per + i % per;
        s = fmaf(cnt[at / V], val[at], s);
      }
    }
    const float mean = lanes_sum(s, lanes) / total;
    if (g < it.ng && lane == 0) part[2 * g] = mean;
  }
  __syncthreads();  // the group means are in part (this block's own writes)
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = int(threadIdx.x) * V + j;
    const int g = it.ty < it.lanes_rows ? (at % used) / per : 0;
    const float d = k[j] - part[2 * g];
    val[at] = n ? fmaf(float(n) * d, d, s2[j]) : 0.f;
  }
  __syncthreads();
  for (int g0 = 0; g0 < it.ng; g0 += step) {
    const int g = g0 + int(threadIdx.x) / lanes;
    float s = 0.f;
    if (g < it.ng) {
      for (int i = lane; i < items; i += lanes) s += val[(i / per) * used + g * per + i % per];
    }
    s = lanes_sum(s, lanes);
    if (g < it.ng && lane == 0) part[2 * g + 1] = s;
  }
}

// mean and rstd of the item's groups from the chunks' sums, into shared memory
template <typename T>
__device__ __forceinline__ void join_stats(const Gn& p, const Item& it, float* gmean,
                                           float* grstd) {
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  const int lanes = lanes_per_group(it.ng);
  const int lane = int(threadIdx.x) % lanes, step = kGnThreads / lanes;
  const float* part = p.part + (it.n * p.chunks * p.groups + it.g0) * 2;
  const long long pitch = (long long)p.groups * 2;
  const float total = float(p.rows) * float(p.per);
  for (int g0 = 0; g0 < it.ng; g0 += step) {
    const int g = g0 + int(threadIdx.x) / lanes;
    float s = 0.f, m2 = 0.f;
    if (g < it.ng) {
      for (int c = lane; c < p.chunks; c += lanes) {
        const float n = float(min(p.chunk_rows, p.rows - c * p.chunk_rows)) * float(p.per);
        s = fmaf(n, part[c * pitch + 2 * g], s);
      }
    }
    const float mean = lanes_sum(s, lanes) / total;  // from the group's first value
    if (g < it.ng) {
      for (int c = lane; c < p.chunks; c += lanes) {
        const float n = float(min(p.chunk_rows, p.rows - c * p.chunk_rows)) * float(p.per);
        const float d = part[c * pitch + 2 * g] - mean;
        m2 += fmaf(n * d, d, part[c * pitch + 2 * g + 1]);
      }
    }
    m2 = lanes_sum(m2, lanes);
    if (g < it.ng && lane == 0) {
      const float rstd = 1.f / sqrtf(m2 / total + p.eps);
      gmean[g] = mean + to_f32(x[(long long)g * p.per]);
      grstd[g] = rstd;
      if (it.chunk == 0) {
        p.mean[it.n * p.groups + it.g0 + g] = gmean[g];
        p.rstd[it.n * p.groups + it.g0 + g] = rstd;
      }
    }
  }
  __syncthreads();
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) k_gn_apply(const Gn p) {
  __shared__ float gmean[kGnThreads * V], grstd[kGnThreads * V];
  const Item it = item_of<V>(p, blockIdx.x);
  join_stats<T>(p, it, gmean, grstd);
  if (it.ty >= it.lanes_rows) return;
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  T* y = static_cast<T*>(p.y) + it.n * p.y_batch + it.c0;
  for (int col = it.tx; col < it.width / V; col += it.cols) {
    float m[V], a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = col * V + j, g = c / p.per;
      const float w = p.weight ? load_as_f32(p.weight, p.param_dtype, it.c0 + c) : 1.f;
      b[j] = p.bias ? load_as_f32(p.bias, p.param_dtype, it.c0 + c) : 0.f;
      m[j] = gmean[g];
      a[j] = grstd[g] * w;
    }
    for (long long r = it.r0 + it.ty; r < it.r1; r += kGnUnroll * it.lanes_rows) {
      Pack<T, V> in[kGnUnroll];
#pragma unroll
      for (int u = 0; u < kGnUnroll; ++u) {
        const long long rr = r + (long long)u * it.lanes_rows;
        if (rr < it.r1) in[u] = load_pack<T, V>(x + rr * p.x_row + (long long)col * V);
      }
#pragma unroll
      for (int u = 0; u < kGnUnroll; ++u) {
        const long long rr = r + (long long)u * it.lanes_rows;
        if (rr >= it.r1) break;
        float v[V];
        unpack(in[u], v);
        Pack<T, V> out;
#pragma unroll
        for (int j = 0; j < V; ++j)
          out.v[j] = from_f32<T>(act_of<ACT>(fmaf(v[j] - m[j], a[j], b[j])));
        *reinterpret_cast<Pack<T, V>*>(y + rr * p.y_row + (long long)col * V) = out;
      }
    }
  }
}

// ------------------------------------------------------------------ backward
// A thread's channel constants.
template <int V>
struct Lane {
  float mean[V], rstd[V], w[V], b[V];
  __device__ __forceinline__ void load(const Gn& p, const Item& it, int col) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = it.c0 + col * V + j, g = c / p.per;
      mean[j] = p.mean[it.n * p.groups + g];
      rstd[j] = p.rstd[it.n * p.groups + g];
      w[j] = p.weight ? load_as_f32(p.weight, p.param_dtype, c) : 1.f;
      b[j] = p.bias ? load_as_f32(p.bias, p.param_dtype, c) : 0.f;
    }
  }
  // h = (x - mean) rstd and e = dy act'(z).  z is formed as in the forward pass, so that a
  // relu cuts where it did there.
  template <int ACT>
  __device__ __forceinline__ void h_and_e(int j, float x, float dy, float* h, float* e) const {
    const float d = x - mean[j];
    *h = d * rstd[j];
    *e = ACT == EFCP_ACT_NONE ? dy : dy * act_grad<ACT>(fmaf(d, rstd[j] * w[j], b[j]));
  }
};

// Per channel and chunk of rows: sum e h, then sum e.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) k_gn_bwd_sums(const Gn p) {
  __shared__ float sh[2][kGnThreads * V];
  const Item it = item_of<V>(p, blockIdx.x);
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  const T* dy = static_cast<const T*>(p.dy) + it.n * p.dy_batch + it.c0;
  float* part = p.part + (it.n * p.chunks + it.chunk) * 2 * p.channels + it.c0;
  // the same rounds for every thread: there is a barrier inside
  for (int col0 = 0; col0 < it.width / V; col0 += it.cols) {
    const int col = col0 + it.tx;
    float eh[V], es[V];
#pragma unroll
    for (int j = 0; j < V; ++j) eh[j] = es[j] = 0.f;
    if (it.ty < it.lanes_rows && col < it.width / V) {
      Lane<V> ln;
      ln.load(p, it, col);
      for (long long r = it.r0 + it.ty; r < it.r1; r += kGnUnroll * it.lanes_rows) {
        Pack<T, V> ax[kGnUnroll], ad[kGnUnroll];
#pragma unroll
        for (int u = 0; u < kGnUnroll; ++u) {
          const long long rr = r + (long long)u * it.lanes_rows;
          if (rr < it.r1) {
            ax[u] = load_pack<T, V>(x + rr * p.x_row + (long long)col * V);
            ad[u] = load_pack<T, V>(dy + rr * p.dy_row + (long long)col * V);
          }
        }
#pragma unroll
        for (int u = 0; u < kGnUnroll; ++u) {
          if (r + (long long)u * it.lanes_rows >= it.r1) break;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float h, e;
            ln.template h_and_e<ACT>(j, to_f32(ax[u].v[j]), to_f32(ad[u].v[j]), &h, &e);
            eh[j] = fmaf(e, h, eh[j]);
            es[j] += e;
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      sh[0][threadIdx.x * V + j] = eh[j];
      sh[1][threadIdx.x * V + j] = es[j];
    }
    __syncthreads();
    const int used = it.cols * V;
    for (int c = threadIdx.x; c < used && col0 * V + c < it.width; c += kGnThreads) {
      float s0 = 0.f, s1 = 0.f;
      for (int t = 0; t < it.lanes_rows; ++t) {
        s0 += sh[0][t * used + c];
        s1 += sh[1][t * used + c];
      }
      part[col0 * V + c] = s0;
      part[p.channels + col0 * V + c] = s1;
    }
    __syncthreads();
  }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) k_gn_bwd_apply(const Gn p) {
  // mean over the group of e w h and of e w
  __shared__ float ghb[kGnThreads * V], gea[kGnThreads * V];
  const Item it = item_of<V>(p, blockIdx.x);
  {
    const int lanes = lanes_per_group(it.ng);
    const int lane = int(threadIdx.x) % lanes, step = kGnThreads / lanes;
    const float* part = p.part + it.n * p.chunks * 2 * p.channels;
    const float total = float(p.rows) * float(p.per);
    for (int g0 = 0; g0 < it.ng; g0 += step) {
      const int g = g0 + int(threadIdx.x) / lanes;
      float sb = 0.f, sa = 0.f;
      if (g < it.ng) {
        for (long long i = lane; i < (long long)p.chunks * p.per; i += lanes) {
          const int c = (it.g0 + g) * p.per + int(i % p.per);
          const float* q = part + (i / p.per) * 2 * p.channels + c;
          const float w = p.weight ? load_as_f32(p.weight, p.param_dtype, c) : 1.f;
          sb = fmaf(w, q[0], sb);
          sa = fmaf(w, q[p.channels], sa);
        }
      }
      sb = lanes_sum(sb, lanes);
      sa = lanes_sum(sa, lanes);
      if (g < it.ng && lane == 0) {
        ghb[g] = sb / total;
        gea[g] = sa / total;
      }
    }
    __syncthreads();
  }
  if (it.ty >= it.lanes_rows) return;
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  const T* dy = static_cast<const T*>(p.dy) + it.n * p.dy_batch + it.c0;
  T* dx = static_cast<T*>(p.y) + it.n * p.y_batch + it.c0;
  for (int col = it.tx; col < it.width / V; col += it.cols) {
    Lane<V> ln;
    ln.load(p, it, col);
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a[j] = gea[(col * V + j) / p.per];
      b[j] = ghb[(col * V + j) / p.per];
    }
    for (long long r = it.r0 + it.ty; r < it.r1; r += kGnUnroll * it.lanes_rows) {
      Pack<T, V> ax[kGnUnroll], ad[kGnUnroll];
#pragma unroll
      for (int u = 0; u < kGnUnroll; ++u) {
        const long long rr = r + (long long)u * it.lanes_rows;
        if (rr < it.r1) {
          ax[u] = load_pack<T, V>(x + rr * p.x_row + (long long)col * V);
          ad[u] = load_pack<T, V>(dy + rr * p.dy_row + (long long)col * V);
        }
      }
#pragma unroll
      for (int u = 0; u < kGnUnroll; ++u) {
        const long long rr = r + (long long)u * it.lanes_rows;
        if (rr >= it.r1) break;
        Pack<T, V> out;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float h, e;
          ln.template h_and_e<ACT>(j, to_f32(ax[u].v[j]), to_f32(ad[u].v[j]), &h, &e);
          out.v[j] = from_f32<T>(ln.rstd[j] * (fmaf(e, ln.w[j], -a[j]) - h * b[j]));
        }
        *reinterpret_cast<Pack<T, V>*>(dx + rr * p.y_row + (long long)col * V) = out;
      }
    }
  }
}

// dweight and dbias: column sums of the chunks' sums, in fp64 and a fixed order.  32 channels per
// block, the rows shared among its warps.
constexpr int kGnSumWarps = 16;
__global__ void __launch_bounds__(32 * kGnSumWarps)
    k_gn_param_grads(const float* __restrict__ part, long long n, int channels, int dtype,
                     void* dweight, void* dbias) {
  __shared__ double sh[2][kGnSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = int(blockIdx.x) * 32 + lane;
  double s0 = 0.0, s1 = 0.0;
  if (c < channels) {
#pragma unroll 4
    for (long long i = warp; i < n; i += kGnSumWarps) {
      s0 += double(part[i * 2 * channels + c]);
      s1 += double(part[(i * 2 + 1) * channels + c]);
    }
  }
  sh[0][warp][lane] = s0;
  sh[1][warp][lane] = s1;
  __syncthreads();
  if (warp < 2 && c < channels) {
    double s = 0.0;
    for (int k = 0; k < kGnSumWarps; ++k) s += sh[warp][k][lane];
    void* out = warp == 0 ? dweight : dbias;
    if (out) store_from_f32(out, dtype, c, float(s));
  }
}

// ------------------------------------------------------------------ host
constexpr int kTypeBytes[3] = {4, 2, 2};

bool valid(const efcp_group_norm* d) {
  if (!d || d->n < 0 || d->rows < 1 || d->channels < 1 || d->groups < 1) return false;
  if (d->channels >= (1ll << 30) || d->channels % d->groups) return false;
  if (d->dtype < 0 || d->dtype > 2 || d->param_dtype < 0 || d->param_dtype > 2) return false;
  if (d->act < 0 || d->act > EFCP_ACT_SILU) return false;
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return false;
  const int64_t most = 1ll << 40;
  if (d->rows > most / d->channels || (d->n && d->rows * d->channels > most / d->n)) return false;
  return true;
}

// Rows and samples of a tensor: strides that keep every offset in 63 bits, rows apart; for an
// output also samples apart (in either order: rows inside samples or samples inside rows).
bool valid_strides(const efcp_group_norm* d, int64_t batch, int64_t row, bool output) {
  const int64_t most = 1ll << 50;
  if (row < d->channels || batch < 0 || row > most / d->rows) return false;
  if (d->n > 1 && batch > most / d->n) return false;
  if (output && d->n > 1) {
    const bool rows_inside = batch >= (d->rows - 1) * row + d->channels;
    const bool samples_inside =
        batch >= d->channels && (d->rows == 1 || row >= (d->n - 1) * batch + d->channels);
    if (!rows_inside && !samples_inside) return false;
  }
  return true;
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

struct Tensor {
  const void* ptr;
  int64_t batch, row;
};

// V is the widest of 16 bytes, 4 bytes and one element that every address is a multiple of and a
// tile of whole groups can be made of; then tiles and chunks.
// How many chunks: enough blocks to fill the GPU (8 per SM), and no thread with more than
// kGnMaxRowsPerThread rows (the bound of k_gn_stats).
int plan(const efcp_group_norm& d, const Tensor* t, int nt, int sms, Gn* p) {
  const int size = kTypeBytes[d.dtype], per = int(d.channels / d.groups);
  p->rows = d.rows;
  p->channels = int(d.channels);
  p->groups = d.groups;
  p->per = per;
  p->param_dtype = d.param_dtype;
  p->eps = d.eps;
  p->x_batch = d.x_batch; p->x_row = d.x_row;
  p->y_batch = d.y_batch; p->y_row = d.y_row;
  p->dy_batch = d.dy_batch; p->dy_row = d.dy_row;
  int v = 1;
  for (int bytes : {16, 4}) {
    const int w = bytes / size;
    if (w < 1 || w == 1) continue;
    bool ok = d.channels % w == 0;
    for (int i = 0; i < nt; ++i)
      ok = ok && reinterpret_cast<uintptr_t>(t[i].ptr) % bytes == 0 && t[i].row % w == 0 &&
           t[i].batch % w == 0;
    const int unit = w / gcd(per, w);  // groups whose channels are a whole number of vectors
    if (ok && (unit == 1 || int64_t(unit) * per / w <= kGnThreads)) {
      v = w;
      break;
    }
  }
  const int unit = v / gcd(per, v);
  const int64_t unit_cols = int64_t(unit) * per / v;
  const int most = int(std::max<int64_t>(1, kGnThreads / unit_cols)) * unit;
  p->tiles = (d.groups + most - 1) / most;
  p->tile_groups = ((d.groups + p->tiles - 1) / p->tiles + unit - 1) / unit * unit;
  p->tiles = (d.groups + p->tile_groups - 1) / p->tile_groups;
  const int64_t cols = std::min<int64_t>(kGnThreads, int64_t(p->tile_groups) * per / v);
  const int64_t lanes_rows = kGnThreads / cols;
  const int64_t rounds = (int64_t(p->tile_groups) * per / v + cols - 1) / cols;
  const int64_t items = std::max<int64_t>(1, d.n * p->tiles);
  int64_t chunks = (int64_t(sms) * kGnBlocksPerSM + items - 1) / items;
  chunks = std::min(chunks, (d.rows + lanes_rows - 1) / lanes_rows);
  const int64_t longest = std::max<int64_t>(1, kGnMaxRowsPerThread / rounds) * lanes_rows;
  chunks = std::max(chunks, (d.rows + longest - 1) / longest);
  p->chunk_rows = (d.rows + chunks - 1) / chunks;
  p->chunks = int((d.rows + p->chunk_rows - 1) / p->chunk_rows);
  return v;
}

// Blocks of a launch; 0 when they exceed what a grid may have.
unsigned blocks_of(const efcp_group_norm& d, const Gn& p) {
  const int64_t b = d.n * p.tiles * p.chunks;
  return b < (1ll << 31) ? unsigned(b) : 0u;
}

int64_t part_floats(const efcp_group_norm& d, const Gn& p, bool backward) {
  return backward ? d.n * p.chunks * 2 * d.channels : d.n * p.chunks * 2 * d.groups;
}

template <typename T, int V, int ACT>
void launch_forward(const Gn& p, unsigned blocks, cudaStream_t st) {
  k_gn_stats<T, V><<<blocks, kGnThreads, 0, st>>>(p);
  k_gn_apply<T, V, ACT><<<blocks, kGnThreads, 0, st>>>(p);
}
template <typename T, int V, int ACT>
void launch_backward(const Gn& p, unsigned blocks, cudaStream_t st) {
  k_gn_bwd_sums<T, V, ACT><<<blocks, kGnThreads, 0, st>>>(p);
  k_gn_bwd_apply<T, V, ACT><<<blocks, kGnThreads, 0, st>>>(p);
}
template <typename T, int V>
void launch(const Gn& p, int act, bool backward, unsigned blocks, cudaStream_t st) {
  switch (act) {
    case EFCP_ACT_NONE:
      backward ? launch_backward<T, V, EFCP_ACT_NONE>(p, blocks, st)
               : launch_forward<T, V, EFCP_ACT_NONE>(p, blocks, st);
      break;
    case EFCP_ACT_RELU:
      backward ? launch_backward<T, V, EFCP_ACT_RELU>(p, blocks, st)
               : launch_forward<T, V, EFCP_ACT_RELU>(p, blocks, st);
      break;
    default:
      backward ? launch_backward<T, V, EFCP_ACT_SILU>(p, blocks, st)
               : launch_forward<T, V, EFCP_ACT_SILU>(p, blocks, st);
  }
}
template <typename T>
void launch_half(const Gn& p, int v, int act, bool backward, unsigned blocks, cudaStream_t st) {
  if (v == 8) launch<T, 8>(p, act, backward, blocks, st);
  else if (v == 2) launch<T, 2>(p, act, backward, blocks, st);
  else launch<T, 1>(p, act, backward, blocks, st);
}
void launch_any(const Gn& p, int dtype, int v, int act, bool backward, unsigned blocks,
                cudaStream_t st) {
  if (dtype == EFCP_BF16) return launch_half<__nv_bfloat16>(p, v, act, backward, blocks, st);
  if (dtype == EFCP_F16) return launch_half<__half>(p, v, act, backward, blocks, st);
  if (v == 4) launch<float, 4>(p, act, backward, blocks, st);
  else launch<float, 1>(p, act, backward, blocks, st);
}

bool misaligned(const void* p, int bytes) {
  return !p || reinterpret_cast<uintptr_t>(p) % unsigned(bytes) != 0;
}

}  // namespace
}  // namespace efcp

using namespace efcp;

extern "C" {

// The chunks depend on the alignment of the tensors, which is not known here: one element per
// access gives the most chunks, wider accesses fewer.
int64_t efcp_group_norm_workspace_bytes(const efcp_group_norm* desc, int32_t backward) {
  if (!valid(desc)) return -1;
  int sms = device_sms();
  if (sms < 1) sms = 148;  // no device: the SM count of a B200
  int64_t most = 0;
  for (uintptr_t align : {16, 4, 2}) {
    Gn p{};
    const Tensor t{reinterpret_cast<const void*>(align), 0, 0};
    plan(*desc, &t, 1, sms, &p);
    most = std::max(most, part_floats(*desc, p, backward != 0));
  }
  return std::max<int64_t>(16, most * 4);
}

int efcp_group_norm_forward(const efcp_group_norm* desc, const void* x, const void* weight,
                            const void* bias, void* y, float* mean, float* rstd, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || !valid_strides(desc, desc->x_batch, desc->x_row, false) ||
      !valid_strides(desc, desc->y_batch, desc->y_row, true))
    return EFCP_EINVAL;
  if (desc->n == 0) return EFCP_OK;
  const int size = kTypeBytes[desc->dtype], psize = kTypeBytes[desc->param_dtype];
  if (misaligned(x, size) || misaligned(y, size) || misaligned(mean, 4) || misaligned(rstd, 4) ||
      misaligned(workspace, 16) || (weight && misaligned(weight, psize)) ||
      (bias && misaligned(bias, psize)))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Gn p{};
  const Tensor t[2] = {{x, desc->x_batch, desc->x_row}, {y, desc->y_batch, desc->y_row}};
  const int v = plan(*desc, t, 2, sms, &p);
  const unsigned blocks = blocks_of(*desc, p);
  if (!blocks) return EFCP_ETOOBIG;
  if (workspace_bytes < part_floats(*desc, p, false) * 4) return EFCP_ENOMEM;
  p.x = x; p.y = y; p.weight = weight; p.bias = bias;
  p.mean = mean; p.rstd = rstd; p.part = static_cast<float*>(workspace);
  launch_any(p, desc->dtype, v, desc->act, false, blocks, static_cast<cudaStream_t>(stream));
  return cudaGetLastError() == cudaSuccess ? EFCP_OK : EFCP_ECUDA;
}

int efcp_group_norm_backward(const efcp_group_norm* desc, const void* dy, const void* x,
                             const float* mean, const float* rstd, const void* weight,
                             const void* bias, void* dx, void* dweight, void* dbias,
                             void* workspace, int64_t workspace_bytes, void* stream) {
  if (!valid(desc) || !valid_strides(desc, desc->x_batch, desc->x_row, false) ||
      !valid_strides(desc, desc->dy_batch, desc->dy_row, false) ||
      !valid_strides(desc, desc->y_batch, desc->y_row, true))
    return EFCP_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int size = kTypeBytes[desc->dtype], psize = kTypeBytes[desc->param_dtype];
  if ((weight && misaligned(weight, psize)) || (bias && misaligned(bias, psize)) ||
      (dweight && misaligned(dweight, psize)) || (dbias && misaligned(dbias, psize)))
    return EFCP_EINVAL;
  if (desc->n == 0) {
    for (void* out : {dweight, dbias})
      if (out && cudaMemsetAsync(out, 0, size_t(desc->channels) * psize, st) != cudaSuccess)
        return EFCP_ECUDA;
    return EFCP_OK;
  }
  if (misaligned(x, size) || misaligned(dy, size) || misaligned(dx, size) ||
      misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(workspace, 16))
    return EFCP_EINVAL;
  const int sms = device_sms();
  if (sms < 1) return EFCP_ECUDA;
  Gn p{};
  const Tensor t[3] = {{x, desc->x_batch, desc->x_row},
                       {dy, desc->dy_batch, desc->dy_row},
                       {dx, desc->y_batch, desc->y_row}};
  const int v = plan(*desc, t, 3, sms, &p);
  const unsigned blocks = blocks_of(*desc, p);
  if (!blocks) return EFCP_ETOOBIG;
  if (workspace_bytes < part_floats(*desc, p, true) * 4) return EFCP_ENOMEM;
  p.x = x; p.dy = dy; p.y = dx; p.weight = weight; p.bias = bias;
  p.mean = const_cast<float*>(mean); p.rstd = const_cast<float*>(rstd);
  p.part = static_cast<float*>(workspace);
  launch_any(p, desc->dtype, v, desc->act, true, blocks, st);
  if (dweight || dbias)
    k_gn_param_grads<<<unsigned((p.channels + 31) / 32), 32 * kGnSumWarps, 0, st>>>(
        p.part, desc->n * p.chunks, p.channels, p.param_dtype, dweight, dbias);
  return cudaGetLastError() == cudaSuccess ? EFCP_OK : EFCP_ECUDA;
}

}  // extern "C"
