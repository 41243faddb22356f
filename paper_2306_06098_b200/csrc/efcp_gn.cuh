// Group normalisation with an activation on channels-last tensors, forward and backward (the
// formulas stand in include/efcp.h).
//
// Memory bounds it: forward x is read and y written once, backward x and dy are read and
// dx is written once.  Both directions need sums over a whole group before the first result, so the
// input has to stay on the chip in between, or is read twice.
//
//   resident   A cluster of up to 16 thread blocks takes one sample's tile of channels and holds all
//              of it in shared memory (about 200 KB per SM in four blocks, so that some load while
//              others compute); the blocks exchange their sums through each other's shared memory.
//              One read, one write.
//   streamed   For samples that do not fit: one pass for the sums of chunks of rows, a small
//              kernel that joins them, one pass for the result.
//
// A tile is a number of whole groups.  In both forms a thread owns V neighbouring channels
// (one access of up to 16 bytes) and walks down rows, so what belongs to a channel - weight,
// bias, statistics, its sums - stays with the thread.
//
// Measured on a B200 (copy rate 6.56 TB/s), device time: 256 x 112 x 112 x 64 bf16 relu forward 199 us,
// 4.1 TB/s; 256 x 56 x 56 x 64 bf16 silu backward 102 us, 3.0 TB/s; 128 x 32 x 32 x 16 fp32 forward 6.2 us;
// 1 x 7 x 7 x 512 fp16 forward 3.4 us; streamed, 1 x 512 x 512 x 128 bf16 silu forward 67 us,
// backward 129 us.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "efcp.h"
#include "efcp_gn.h"
#include "efcp_launch.cuh"
#include "efcp_num.cuh"

namespace efcp {
namespace {

namespace cg = cooperative_groups;

static_assert(kGnSmemOf2 <= int64_t(kMaxDynamicSmem), "what a launch may ask for");

// What a thread block works on.
struct Item {
  long long n, r0, r1;           // sample, rows r0 .. r1 of it (none when r1 <= r0)
  int chunk, g0, ng, c0, width;  // groups g0 .. g0 + ng, channels c0 .. c0 + width
  int tx, ty;                    // this thread's place among the accesses side by side
  bool on;                       // whether that place exists
};

// `chunk`: the chunk of the sample's tile, `q`: the tile among those of all samples.
template <int V>
__device__ __forceinline__ Item item_of(const Gn& p, unsigned chunk, unsigned q) {
  Item it;
  it.chunk = int(chunk);
  unsigned s = q, tile = 0;
  if (p.tiles > 1) {
    s = q / unsigned(p.tiles);
    tile = q - s * unsigned(p.tiles);
  }
  it.n = s;
  it.r0 = it.chunk * p.chunk_rows;
  it.r1 = min(p.rows, it.r0 + p.chunk_rows);
  it.g0 = int(tile) * p.tile_groups;
  it.ng = min(p.tile_groups, p.groups - it.g0);
  it.c0 = it.g0 * p.per;
  it.width = it.ng * p.per;
  if (p.pitch_log >= 0) {
    it.ty = int(threadIdx.x) >> p.pitch_log;
    it.tx = int(threadIdx.x) & ((1 << p.pitch_log) - 1);
  } else {
    it.ty = int(threadIdx.x) / p.cols;
    it.tx = int(threadIdx.x) - it.ty * p.cols;
  }
  it.on = it.tx * V < it.width && it.ty < p.lanes_rows;
  return it;
}

// V elements through the read-only path (the input is not written during the launch, so loads
// may move ahead of the stores of earlier rows).
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

// V fp32 values, two to an instruction where there are two (sm_100's packed fp32 arithmetic: the
// same rounding as one by one, at half the instructions).
template <int V>
struct Vec {
  float v[V];
};
template <int V>
__device__ __forceinline__ Vec<V> fill(float x) {
  Vec<V> r;
#pragma unroll
  for (int j = 0; j < V; ++j) r.v[j] = x;
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> fma(const Vec<V>& a, const Vec<V>& b, const Vec<V>& c) {
  Vec<V> r;
  if constexpr (V == 1) {
    r.v[0] = fmaf(a.v[0], b.v[0], c.v[0]);
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const float2 t = __ffma2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]),
                                  make_float2(c.v[j], c.v[j + 1]));
      r.v[j] = t.x;
      r.v[j + 1] = t.y;
    }
  }
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> operator+(const Vec<V>& a, const Vec<V>& b) {
  Vec<V> r;
  if constexpr (V == 1) {
    r.v[0] = a.v[0] + b.v[0];
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const float2 t =
          __fadd2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]));
      r.v[j] = t.x;
      r.v[j + 1] = t.y;
    }
  }
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> operator*(const Vec<V>& a, const Vec<V>& b) {
  Vec<V> r;
  if constexpr (V == 1) {
    r.v[0] = a.v[0] * b.v[0];
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const float2 t =
          __fmul2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]));
      r.v[j] = t.x;
      r.v[j + 1] = t.y;
    }
  }
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> minus(Vec<V> a) {
#pragma unroll
  for (int j = 0; j < V; ++j) a.v[j] = -a.v[j];
  return a;
}

template <typename T, int V>
__device__ __forceinline__ Vec<V> unpack(const Pack<T, V>& a) {
  Vec<V> r;
#pragma unroll
  for (int j = 0; j < V; ++j) r.v[j] = to_f32(a.v[j]);
  return r;
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack(const Vec<V>& a) {
  Pack<T, V> r;
#pragma unroll
  for (int j = 0; j < V; ++j) r.v[j] = from_f32<T>(a.v[j]);
  return r;
}

// max(a, b), NaN when either is one
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 1 / x by the hardware: 0 for an infinite x
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// 2^x by the hardware
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float weight_of(const Gn& p, int c) {
  return p.weight ? load_as_f32(p.weight, p.param_dtype, c) : 1.f;
}
__device__ __forceinline__ float bias_of(const Gn& p, int c) {
  return p.bias ? load_as_f32(p.bias, p.param_dtype, c) : 0.f;
}

// Sum over groups of neighbouring lanes (a power of two of them), the same in all of them.
template <typename F>
__device__ __forceinline__ F lanes_sum(F v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// 1 / (1 + exp(-z)) with the hardware's reciprocal and power of two, each within 2 units in the last place.
// The power's argument is rounded to fp32, so exp(-z) is off by up to another |z| units or so; where that is many, z
// far below 0, the result is small.  0 where exp(-z) overflows.
template <int V>
__device__ __forceinline__ Vec<V> sigmoid_of(const Vec<V>& z) {
  Vec<V> t = z * fill<V>(-1.44269504f);
#pragma unroll
  for (int j = 0; j < V; ++j) t.v[j] = exp2_fast(t.v[j]);
  t = t + fill<V>(1.f);
#pragma unroll
  for (int j = 0; j < V; ++j) t.v[j] = rcp_fast(t.v[j]);
  return t;
}
// act(z)
template <int ACT, int V>
__device__ __forceinline__ Vec<V> act_of(Vec<V> z) {
  if (ACT == EFCP_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < V; ++j) z.v[j] = max_nan(z.v[j], 0.f);
  }
  if (ACT == EFCP_ACT_SILU) z = z * sigmoid_of(z);
  return z;
}
// dy act'(z).  relu's derivative selects: what arrives where it is 0 does not matter, infinite or not.
template <int ACT, int V>
__device__ __forceinline__ Vec<V> through_act(Vec<V> dy, const Vec<V>& z) {
  if (ACT == EFCP_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < V; ++j) dy.v[j] = z.v[j] <= 0.f ? 0.f : dy.v[j];
  }
  if (ACT == EFCP_ACT_SILU) {
    const Vec<V> s = sigmoid_of(z);
    dy = dy * (s * fma(z, fma(s, fill<V>(-1.f), fill<V>(1.f)), fill<V>(1.f)));
  }
  return dy;
}

// ------------------------------------------------------------------ sums inside a block
// Sums a thread's N values over the rows side by side, as far as a warp reaches, and stores
// them in val: p.val_rows rows of p.cols * N values.  Threads that are not `on` bring zeros.
// The caller synchronises.
template <int N>
__device__ __forceinline__ void sum_rows(const Gn& p, const Item& it, const float* v, float* val) {
  float s[N];
#pragma unroll
  for (int j = 0; j < N; ++j) s[j] = v[j];
  if (p.pitch_log < 0) {
    if (it.ty < p.lanes_rows) {
#pragma unroll
      for (int j = 0; j < N; ++j) val[(it.ty * p.cols + it.tx) * N + j] = s[j];
    }
    return;
  }
  for (int o = 1 << p.pitch_log; o < 32; o *= 2) {
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] += __shfl_xor_sync(0xFFFFFFFFu, s[j], o);
  }
  const int warp = int(threadIdx.x) >> 5, lane = int(threadIdx.x) & 31;
  if (lane < p.cols) {
#pragma unroll
    for (int j = 0; j < N; ++j) val[(warp * p.cols + lane) * N + j] = s[j];
  }
}

// Mean and sum of squared deviations M2 of `cnt` values per channel.  Parts are joined by
//     mean = sum n_i mean_i / sum n_i,   M2 = sum M2_i + n_i (mean_i - mean)^2,
// sums without cancellation whatever the data.  The means are held and joined in 64 bits: every join in
// fp32 would round by up to half a unit of the parts' distance from each other, and a chain of them is
// further off than one sum over the group in fp32 (128 x 32 x 32 x 16 fp32: mean and y off by 2.3e-7 with fp32
// joins, 6.7e-8 now; it cost the small calls 0.3 us on the device, 6.0 for 5.7 there).
template <int V>
struct Stats {
  double mean[V];
  Vec<V> q;  // M2
  float cnt;
};

// A thread's own values: sums of d = x - k and of d^2 over n of them, then M2 = sum d^2 - (sum d)^2 / n.
// The subtraction loses what the squares' sum is larger than M2, a factor of 1 + n (k - mean)^2 / M2,
// so k has to be near the mean whatever the data.  With k a mean of c of the values, (k - mean)^2 is at most
// M2 / c, and the factor at most 1 + n / c: 9 on chip (n <= 32 and c = 4, n <= 64 and c = 8).  (k the first value: up to n + 1, rstd
// off by 520 units of 2^-24 where columns of 64 values begin with one far from the rest.)

// M2 of n values from those sums; `inv` = 1 / n.
__device__ __forceinline__ float m2_of(float s1, float s2, float inv) {
  return fmaxf(0.f, fmaf(-(s1 * inv), s1, s2));
}

template <int V>
__device__ __forceinline__ Stats<V> stats_of(int n, const Vec<V>& k, const Vec<V>& s1,
                                             const Vec<V>& s2) {
  Stats<V> s;
  s.cnt = float(n);
  const double inv = n ? 1.0 / double(n) : 0.0;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s.mean[j] = __fma_rn(double(s1.v[j]), inv, double(k.v[j]));
    s.q.v[j] = m2_of(s1.v[j], s2.v[j], float(inv));
  }
  return s;
}

// The same for values that come a batch at a time: segments of at most twice as many values as came before,
// each around the mean so far (a factor of 3 at most), joined one after another.  Segments end at 64
// values, so that the sums of a long run (a group wider than the block) stay short too.  The mean is kept with
// what its rounding to fp32 leaves: without that, rstd was off by 190 units for values 10^5 deviations from zero.
template <int V>
struct Running {
  Vec<V> neg = fill<V>(0.f);  // minus the mean of the n values joined, rounded to fp32,
  Vec<V> rest = neg;          // and what that leaves of it
  Vec<V> q = neg, s1 = neg, s2 = neg;
  int n = 0, open = 0;  // values joined, of the segment

  // m > 0 of the U values of a batch exist.
  template <typename T, int U>
  __device__ __forceinline__ void add(const Pack<T, V> (&a)[U], int m) {
    if (n == 0) {  // the first segment is this batch, around its own mean
      const Vec<V> first = minus(unpack(a[0]));
      Vec<V> s = fill<V>(0.f);
#pragma unroll
      for (int u = 1; u < U; ++u)
        if (u < m) s = s + (unpack(a[u]) + first);
      neg = fma(s, fill<V>(-rcp_fast(float(m))), first);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u < m) {
        const Vec<V> d = unpack(a[u]) + neg;
        s1 = s1 + d;
        s2 = fma(d, d, s2);
      }
    }
    open += m;
    if (open >= min(64, 2 * n)) join();
  }
  __device__ __forceinline__ void join() {
    if (open == 0) return;
    const float inv = rcp_fast(float(open)), w = float(open) * rcp_fast(float(n + open));
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = fmaf(s1.v[j], inv, -rest.v[j]);  // the segment's mean, less the mean so far
      q.v[j] += fmaf(float(n) * w * d, d, m2_of(s1.v[j], s2.v[j], inv));
      const float up = fmaf(w, d, rest.v[j]), old = neg.v[j];
      neg.v[j] = old - up;
      rest.v[j] = up - (old - neg.v[j]);
    }
    s1 = s2 = fill<V>(0.f);
    n += open;
    open = 0;
  }
  __device__ __forceinline__ Stats<V> done() {
    join();
    Stats<V> s;
    s.cnt = float(n);
    s.q = q;
#pragma unroll
    for (int j = 0; j < V; ++j) s.mean[j] = double(rest.v[j]) - double(neg.v[j]);
    return s;
  }
};

// Neighbouring channels of one group joined.
template <int V>
__device__ __forceinline__ Stats<V / 2> fold_once(const Stats<V>& s) {
  Stats<V / 2> r;
  r.cnt = 2.f * s.cnt;
#pragma unroll
  for (int j = 0; j < V / 2; ++j) {
    const float d = float(s.mean[2 * j + 1] - s.mean[2 * j]);
    r.mean[j] = 0.5 * (s.mean[2 * j] + s.mean[2 * j + 1]);
    r.q.v[j] = fmaf(0.5f * s.cnt * d, d, s.q.v[2 * j] + s.q.v[2 * j + 1]);
  }
  return r;
}

// Joins the rows side by side as far as a warp reaches and stores what results in shared memory: p.val_rows
// rows of p.folded_cols values each of the means (64 bits), of M2 and of the counts.
template <int V>
__device__ __forceinline__ void store_stats(const Gn& p, const Item& it, Stats<V> s, float* val) {
  int row = it.ty, col = it.tx;
  bool store = it.ty < p.lanes_rows;
  if (p.pitch_log >= 0) {
    const int lane = int(threadIdx.x) & 31;
    row = int(threadIdx.x) >> 5;
    store = lane < p.cols;
    float all = s.cnt;
    for (int o = 1 << p.pitch_log; o < 32; o *= 2) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    const double inv = all > 0.f ? 1.0 / double(all) : 0.0;
    double sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = double(s.cnt) * s.mean[j];
    for (int o = 1 << p.pitch_log; o < 32; o *= 2) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], o);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const double mean = sum[j] * inv;
      const float d = float(s.mean[j] - mean);
      s.q.v[j] = fmaf(s.cnt * d, d, s.q.v[j]);
      s.mean[j] = mean;
    }
    for (int o = 1 << p.pitch_log; o < 32; o *= 2) {
#pragma unroll
      for (int j = 0; j < V; ++j) s.q.v[j] += __shfl_xor_sync(0xFFFFFFFFu, s.q.v[j], o);
    }
    s.cnt = all;
  }
  if (store) {
    const int at = row * p.folded_cols + col * V;
    double* mean = reinterpret_cast<double*>(val) + at;
    float *q = val + 2 * p.val_floats + at, *n = q + p.val_floats;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      mean[j] = s.mean[j];
      q[j] = s.q.v[j];
      n[j] = s.cnt;
    }
  }
}
template <int V>
__device__ __forceinline__ void fold_stats(const Gn& p, const Item& it, const Stats<V>& s,
                                           int fold, float* val) {
  if constexpr (V == 1) {
    store_stats(p, it, s, val);
  } else {
    if (fold == 1) store_stats(p, it, s, val);
    else fold_stats(p, it, fold_once(s), fold >> 1, val);
  }
}

// Mean and M2 of group g over the block, from what store_stats left (the caller has
// synchronised): the same in all of the group's lanes.  `rows`: of the block.
struct Joined {
  double mean;
  float q;
};
__device__ __forceinline__ Joined group_stats(const Gn& p, int g, bool exists, float rows,
                                              const float* val) {
  const int lanes = 1 << p.lanes_log, lane = int(threadIdx.x) & (lanes - 1);
  const int per = p.folded_per, used = p.folded_cols;
  // lanes over a row's values, or over the rows
  const bool along = per >= lanes;
  const int d0 = along ? lane : 0, dstep = along ? lanes : 1;
  const int t0 = along ? 0 : lane, tstep = along ? 1 : lanes;
  const double* mean = reinterpret_cast<const double*>(val) + g * per;
  const float *q = val + 2 * p.val_floats + g * per, *n = q + p.val_floats;
  double sum = 0.0;
  if (exists) {
    for (int t = t0; t < p.val_rows; t += tstep)
      for (int d = d0; d < per; d += dstep)
        sum = __fma_rn(double(n[t * used + d]), mean[t * used + d], sum);
  }
  sum = lanes_sum(sum, lanes);
  Joined s;
  s.mean = rows > 0.f ? sum / (double(rows) * double(p.per)) : 0.0;
  float m2 = 0.f;
  if (exists) {
    for (int t = t0; t < p.val_rows; t += tstep) {
      for (int d = d0; d < per; d += dstep) {
        const float e = float(mean[t * used + d] - s.mean);
        m2 += fmaf(n[t * used + d] * e, e, q[t * used + d]);
      }
    }
  }
  s.q = lanes_sum(m2, lanes);
  return s;
}

// The group of lane j of an access at column tx, counted from the tile's first: one division.
struct GroupWalk {
  int g, left;  // group; channels left in it, this one included
  __device__ __forceinline__ GroupWalk(int c, int per) : g(c / per), left(per - c % per) {}
  __device__ __forceinline__ void next(int per) {
    if (--left == 0) {
      ++g;
      left = per;
    }
  }
};

// Per-group values of the channels of an access at channel c of the tile.
template <int V>
__device__ __forceinline__ Vec<V> of_groups(const float* values, int c, int per) {
  Vec<V> r;
  GroupWalk w(c, per);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    r.v[j] = values[w.g];
    w.next(per);
  }
  return r;
}
// Values of V channels from a 16-byte aligned array in shared memory, c a multiple of V.
template <int V>
__device__ __forceinline__ Vec<V> of_channels(const float* values, int c) {
  constexpr int Q = V < 4 ? V : 4;
  Vec<V> r;
#pragma unroll
  for (int h = 0; h < V; h += Q) {
    const Pack<float, Q> q = *reinterpret_cast<const Pack<float, Q>*>(values + c + h);
#pragma unroll
    for (int j = 0; j < Q; ++j) r.v[h + j] = q.v[j];
  }
  return r;
}
// The place of a block in its cluster, and of the cluster in the grid.
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_index() {
  unsigned r;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
  return r;
}
// The cluster's barrier where nothing is handed over: a block that has read the others' sums
// arrives, and waits before it ends, since its own may still be read.
__device__ __forceinline__ void leave_arrive() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void leave_wait() {
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// This thread's number of rows of the item.
__device__ __forceinline__ int rows_of_thread(const Gn& p, const Item& it) {
  const int rows = int(it.r1 - it.r0) - it.ty;
  if (!it.on || rows <= 0) return 0;
  if (p.pitch_log >= 0) return (rows + p.lanes_rows - 1) >> p.lanes_rows_log;
  return (rows + p.lanes_rows - 1) / p.lanes_rows;
}

// ------------------------------------------------------------------ resident: shared memory
// Copies one access from global to shared memory without passing through registers, where the
// hardware has a copy of that size (4, 8, 16 bytes).
template <typename T, int V>
__device__ __forceinline__ void copy_in(void* dst, const T* src) {
  if constexpr (sizeof(T) * V == 2) {
    *static_cast<unsigned short*>(dst) = __ldg(reinterpret_cast<const unsigned short*>(src));
  } else {
    const unsigned d = static_cast<unsigned>(__cvta_generic_to_shared(dst));
    if constexpr (sizeof(T) * V == 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(src) : "memory");
  }
}
// Waits for this thread's copies.  (Every thread reads only what it has copied itself.)
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// ------------------------------------------------------------------ resident, forward
// The channels of group g get minus the mean and rstd times the weight; `lane` of `lanes` threads.
__device__ __forceinline__ void finish_group(const Gn& p, const Item& it, int g, float mean,
                                             float m2, float* cmean, float* wei, int lane,
                                             int lanes) {
  const float rstd = rsqrtf(m2 * p.inv_total + p.eps);
  for (int k = g * p.per + lane; k < (g + 1) * p.per; k += lanes) {
    cmean[k] = -mean;
    wei[k] *= rstd;
  }
  if (it.chunk == 0 && lane == 0) {
    p.mean[it.n * p.groups + it.g0 + g] = mean;
    p.rstd[it.n * p.groups + it.g0 + g] = rstd;
  }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 4) k_gn_resident_fwd(const Gn p) {
  extern __shared__ __align__(32) float sm[];
  const int wide = (p.tile_groups * p.per + 3) & ~3, tg = (p.tile_groups + 3) & ~3;
  float* val = sm;
  float* cmean = val + 4 * p.val_floats;  // per channel: minus the mean,
  float* wei = cmean + wide;              // the weight, later times rstd,
  float* bia = wei + wide;                // the bias
  // per group the block's mean and M2, read by the others
  double* bm = reinterpret_cast<double*>(bia + wide);
  float* bq = reinterpret_cast<float*>(bm + tg);
  // [row of this thread] [thread] of V elements
  Pack<T, V>* data = reinterpret_cast<Pack<T, V>*>(bq + tg) + int(threadIdx.x);
  const Item it = item_of<V>(p, cluster_rank(), cluster_index());
  take_turn();
  const int mine = rows_of_thread(p, it);
  const int c = it.tx * V;
  {
    const T* px = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0 +
                  (it.r0 + it.ty) * p.x_row + c;
    const long long step = p.lanes_rows * p.x_row;
#pragma unroll 4
    for (int k = 0; k < mine; ++k, px += step) copy_in<T, V>(data + k * kGnThreads, px);
  }
  for (int k = threadIdx.x; k < it.width; k += kGnThreads) {
    wei[k] = weight_of(p, it.c0 + k);
    bia[k] = bias_of(p, it.c0 + k);
  }
  copies_done();
  {
    Vec<V> centre = fill<V>(0.f), s1 = centre, s2 = centre;
    if (mine) {
      // of 4 rows, of 8 where there are more than 32, spread over the thread's (fewer come twice)
      const int some = mine > 32 ? 3 : 2;
      const Vec<V> first = unpack(data[0]), from = minus(first);
      for (int h = 0; h < (mine > 1 ? 1 << some : 0); h += 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          s1 = s1 + (unpack(data[((h + k) * mine >> some) * kGnThreads]) + from);
      }
      centre = fma(s1, fill<V>(some == 3 ? 0.125f : 0.25f), first);
      s1 = fill<V>(0.f);
      const Vec<V> neg = minus(centre);
#pragma unroll 4
      for (int k = 0; k < mine; ++k) {
        const Vec<V> d = unpack(data[k * kGnThreads]) + neg;
        s1 = s1 + d;
        s2 = fma(d, d, s2);
      }
    }
    fold_stats(p, it, stats_of(mine, centre, s1, s2), p.fold, val);
  }
  __syncthreads();
  cg::cluster_group cluster = cg::this_cluster();
  const float rows = float(max(0, int(it.r1 - it.r0)));
  const int lanes = 1 << p.lanes_log, lane = int(threadIdx.x) & (lanes - 1);
  for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.lanes_log) {
    const int g = g0 + (int(threadIdx.x) >> p.lanes_log);
    const Joined s = group_stats(p, g, g < it.ng, rows, val);
    if (g < it.ng) {
      if (p.chunks == 1) {
        finish_group(p, it, g, float(s.mean), s.q, cmean, wei, lane, lanes);
      } else if (lane == 0) {
        bm[g] = s.mean;
        bq[g] = s.q;
      }
    }
  }
  if (p.chunks > 1) {
    cluster.sync();
    // a group's blocks are joined by neighbouring lanes, one each
    const int links = 1 << p.links_log, r = int(threadIdx.x) & (links - 1);
    const float have =
        float(max(0, min(int(p.chunk_rows), int(p.rows) - r * int(p.chunk_rows))));
    for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.links_log) {
      const int g = g0 + (int(threadIdx.x) >> p.links_log);
      double m = 0.0;
      float q = 0.f;
      const bool there = g < it.ng && r < p.chunks && have > 0.f;
      if (there) {
        m = cluster.map_shared_rank(bm, r)[g];
        q = cluster.map_shared_rank(bq, r)[g];
      }
      const double mean = lanes_sum(there ? double(have) * m : 0.0, links) * p.inv_rows;
      const float d = float(m - mean);
      q = lanes_sum(there ? fmaf(have * float(p.per) * d, d, q) : 0.f, links);
      if (g < it.ng) finish_group(p, it, g, float(mean), q, cmean, wei, r, links);
    }
  }
  __syncthreads();
  if (p.chunks > 1) leave_arrive();
  if (mine) {
    const Vec<V> m = of_channels<V>(cmean, c), f = of_channels<V>(wei, c);
    const Vec<V> b = of_channels<V>(bia, c);
    T* py = static_cast<T*>(p.y) + it.n * p.y_batch + it.c0 + (it.r0 + it.ty) * p.y_row + c;
    const long long step = p.lanes_rows * p.y_row;
#pragma unroll 4
    for (int k = 0; k < mine; ++k, py += step)
      *reinterpret_cast<Pack<T, V>*>(py) =
          pack<T, V>(act_of<ACT>(fma(unpack(data[k * kGnThreads]) + m, f, b)));
  }
  if (p.chunks > 1) leave_wait();
}

// ------------------------------------------------------------------ resident, backward
// Per channel P = sum e h and Q = sum e over the block's rows, from them the group's sums of
// e w h and e w over the cluster, then dx = rstd (e w - mean(e w) - h mean(e w h)).  The channels'
// sums of the whole sample go to `part` for dweight and dbias.
//
// x and dy stay in shared memory and e is computed in both passes: an e in fp32 in the place of dy
// would spare the second pass silu's two special functions per element, but halves the rows a
// thread has room for, and few rows do not pay for the sums in between (184 us with it, 107 us without, for
// 256 x 56 x 56 x 64 bf16 with silu, when this was tried; 102 us since).  silu's exponential and
// reciprocal keep the special function units half busy, twice per element.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 4) k_gn_resident_bwd(const Gn p) {
  using P = Pack<T, V>;
  extern __shared__ __align__(32) float sm[];
  const int wide = (p.tile_groups * p.per + 3) & ~3, tg = (p.tile_groups + 3) & ~3;
  float* val0 = sm;
  float* val1 = val0 + p.val_floats;
  float* wei = val1 + p.val_floats;  // per channel: weight,
  float* bia = wei + wide;     // bias,
  float* cm = bia + wide;      // minus the mean,
  float* cr = cm + wide;       // rstd,
  float* tot0 = cr + wide;     // P and Q of this block,
  float* tot1 = tot0 + wide;
  float* cqb = tot1 + wide;    // and minus rstd times the group's means of e w h and of e w
  float* cqa = cqb + wide;
  float* gb = cqa + wide;      // per group: sums of e w h and of e w of this block
  float* ga = gb + tg;
  float* data = ga + tg;
  const Item it = item_of<V>(p, cluster_rank(), cluster_index());
  take_turn();
  const int mine = rows_of_thread(p, it);
  // x, then dy: [row of this thread] [thread] of V elements
  P* xs = reinterpret_cast<P*>(data) + int(threadIdx.x);
  P* ds = xs + p.thread_rows * kGnThreads;
  const long long row = it.r0 + it.ty;
  const int c = it.tx * V, at = it.c0 + c;
  {
    const T* px = static_cast<const T*>(p.x) + it.n * p.x_batch + row * p.x_row + at;
    const T* pd = static_cast<const T*>(p.dy) + it.n * p.dy_batch + row * p.dy_row + at;
    const long long xstep = p.lanes_rows * p.x_row, dstep = p.lanes_rows * p.dy_row;
#pragma unroll 4
    for (int k = 0; k < mine; ++k, px += xstep, pd += dstep) {
      copy_in<T, V>(xs + k * kGnThreads, px);
      copy_in<T, V>(ds + k * kGnThreads, pd);
    }
  }
  for (int k = threadIdx.x; k < it.width; k += kGnThreads) {
    const long long g = it.n * p.groups + it.g0 + k / p.per;
    wei[k] = weight_of(p, it.c0 + k);
    bia[k] = bias_of(p, it.c0 + k);
    cm[k] = -p.mean[g];
    cr[k] = p.rstd[g];
  }
  __syncthreads();
  copies_done();
  Vec<V> s0 = fill<V>(0.f), s1 = s0;
  if (mine) {
    const Vec<V> m = of_channels<V>(cm, c), b = of_channels<V>(bia, c);
    const Vec<V> f = of_channels<V>(cr, c) * of_channels<V>(wei, c);
#pragma unroll 4
    for (int k = 0; k < mine; ++k) {
      const Vec<V> u = unpack(xs[k * kGnThreads]) + m;
      Vec<V> e = unpack(ds[k * kGnThreads]);
      if (ACT != EFCP_ACT_NONE) e = through_act<ACT>(e, fma(u, f, b));
      s0 = fma(e, u, s0);
      s1 = s1 + e;
    }
    s0 = s0 * of_channels<V>(cr, c);
  }
  sum_rows<V>(p, it, s0.v, val0);
  sum_rows<V>(p, it, s1.v, val1);
  __syncthreads();
  cg::cluster_group cluster = cg::this_cluster();
  const int used = p.cols * V;
  const bool grads = p.dweight || p.dbias;
  float* part = p.part + it.n * 2 * p.channels + it.c0;
  {
    const int lanes = 1 << p.lanes_log, lane = int(threadIdx.x) & (lanes - 1);
    const bool along = p.per >= lanes;  // lanes over a row's values, or over the rows
    const int d0 = along ? lane : 0, dstep = along ? lanes : 1;
    const int t0 = along ? 0 : lane, tstep = along ? 1 : lanes;
    for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.lanes_log) {
      const int g = g0 + (int(threadIdx.x) >> p.lanes_log);
      float sb = 0.f, sa = 0.f;
      if (g < it.ng) {
        for (int d = g * p.per + d0; d < (g + 1) * p.per; d += dstep) {
          float t1 = 0.f, t2 = 0.f;
          for (int t = t0; t < p.val_rows; t += tstep) {
            t1 += val0[t * used + d];
            t2 += val1[t * used + d];
          }
          sb = fmaf(wei[d], t1, sb);
          sa = fmaf(wei[d], t2, sa);
        }
      }
      sb = lanes_sum(sb, lanes);
      sa = lanes_sum(sa, lanes);
      if (g < it.ng) {
        if (p.chunks == 1) {
          for (int k = g * p.per + lane; k < (g + 1) * p.per; k += lanes) {
            cqb[k] = -cr[k] * (sb * p.inv_total);
            cqa[k] = -cr[k] * (sa * p.inv_total);
          }
        } else if (lane == 0) {
          gb[g] = sb;
          ga[g] = sa;
        }
      }
    }
  }
  if (grads) {
    // (from the far end: the first threads have the groups' sums to form)
    for (int k = kGnThreads - 1 - int(threadIdx.x); k < it.width; k += kGnThreads) {
      float t0 = 0.f, t1 = 0.f;
#pragma unroll 4
      for (int t = 0; t < p.val_rows; ++t) {
        t0 += val0[t * used + k];
        t1 += val1[t * used + k];
      }
      if (p.chunks == 1) {
        part[k] = t0;
        part[p.channels + k] = t1;
      } else {
        tot0[k] = t0;
        tot1[k] = t1;
      }
    }
  }
  if (p.chunks > 1) {
    cluster.sync();
    // a group's blocks are joined by neighbouring lanes, one each
    const int links = 1 << p.links_log, r = int(threadIdx.x) & (links - 1);
    for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.links_log) {
      const int g = g0 + (int(threadIdx.x) >> p.links_log);
      float sb = 0.f, sa = 0.f;
      if (g < it.ng && r < p.chunks) {
        sb = cluster.map_shared_rank(gb, r)[g];
        sa = cluster.map_shared_rank(ga, r)[g];
      }
      sb = lanes_sum(sb, links) * p.inv_total;
      sa = lanes_sum(sa, links) * p.inv_total;
      if (g < it.ng) {
        for (int k = g * p.per + r; k < (g + 1) * p.per; k += links) {
          cqb[k] = -cr[k] * sb;
          cqa[k] = -cr[k] * sa;
        }
      }
    }
    if (grads) {  // each block of the cluster joins its share of the channels
      const int share = (it.width + p.chunks - 1) / p.chunks;
      const int c1 = min(it.width, (it.chunk + 1) * share);
      for (int k = it.chunk * share + kGnThreads - 1 - int(threadIdx.x); k < c1; k += kGnThreads) {
        float t0 = 0.f, t1 = 0.f;
#pragma unroll 4
        for (int q = 0; q < p.chunks; ++q) {
          t0 += cluster.map_shared_rank(tot0, q)[k];
          t1 += cluster.map_shared_rank(tot1, q)[k];
        }
        part[k] = t0;
        part[p.channels + k] = t1;
      }
    }
  }
  __syncthreads();
  if (p.chunks > 1) leave_arrive();
  if (mine) {
    const Vec<V> m = of_channels<V>(cm, c), rs = of_channels<V>(cr, c);
    const Vec<V> f = rs * of_channels<V>(wei, c), b = of_channels<V>(bia, c);
    const Vec<V> qa = of_channels<V>(cqa, c), qb = of_channels<V>(cqb, c);
    T* po = static_cast<T*>(p.y) + it.n * p.y_batch + row * p.y_row + at;
    const long long step = p.lanes_rows * p.y_row;
#pragma unroll 4
    for (int k = 0; k < mine; ++k, po += step) {
      const Vec<V> u = unpack(xs[k * kGnThreads]) + m;
      Vec<V> e = unpack(ds[k * kGnThreads]);
      if (ACT != EFCP_ACT_NONE) e = through_act<ACT>(e, fma(u, f, b));
      *reinterpret_cast<P*>(po) = pack<T, V>(fma(u * rs, qb, fma(e, f, qa)));
    }
  }
  if (p.chunks > 1) leave_wait();
}

// ------------------------------------------------------------------ streamed
// Bound by memory in the two passes (20 and 31 us of 1 x 512 x 512 x 128 bf16 forward, 58 and 67 us backward, where
// silu takes its share again) and by latency in the joins (15 and 8 us: 592 chunks, few columns).
// Accesses in flight per thread and input: about 32 registers' worth.
template <typename T, int V>
constexpr int kAhead = sizeof(T) * V == 16 ? 4 : 8;

// (Six blocks an SM, as k_gn_apply has, would spill here: 68 us against 65.5 for the call above when it was tried.)
// The statistics of every group over a chunk of rows: the mean as two floats (its fp32 value and what
// that leaves) and M2, one after another.
template <typename T, int V>
__global__ void __launch_bounds__(kGnThreads, 5) k_gn_stats(const Gn p) {
  constexpr int U = kAhead<T, V>;
  extern __shared__ __align__(32) float sm[];
  float* val = sm;
  const Item it = item_of<V>(p, blockIdx.x % unsigned(p.chunks), blockIdx.x / unsigned(p.chunks));
  take_turn();
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  Running<V> sums;
  if (it.on) {
    // (more than one round only where a single group is wider than the block)
    for (int c = it.tx; c < it.width / V; c += p.cols) {
      for (long long r = it.r0 + it.ty; r < it.r1; r += U * p.lanes_rows) {
        Pack<T, V> a[U];
        int m = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long rr = r + (long long)u * p.lanes_rows;
          if (rr < it.r1) {
            a[u] = load_pack<T, V>(x + rr * p.x_row + (long long)c * V);
            m = u + 1;
          }
        }
        sums.add(a, m);
      }
    }
  }
  fold_stats(p, it, sums.done(), p.fold, val);
  __syncthreads();
  float* part = p.part + ((it.n * p.chunks + it.chunk) * p.groups + it.g0) * 3;
  for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.lanes_log) {
    const int g = g0 + (int(threadIdx.x) >> p.lanes_log);
    const Joined s = group_stats(p, g, g < it.ng, float(it.r1 - it.r0), val);
    if (g < it.ng && (int(threadIdx.x) & ((1 << p.lanes_log) - 1)) == 0) {
      part[3 * g] = float(s.mean);
      part[3 * g + 1] = float(s.mean - double(part[3 * g]));
      part[3 * g + 2] = s.q;
    }
  }
}

// The kernels between the two passes: 32 columns (groups, channels) per block, the rows shared among its
// warps, so that loads of neighbouring columns are loads of neighbouring addresses.
constexpr int kGnSumWarps = 32;

// Sum over the block's warps of their lane's value, in a fixed order, the same in all of them.
template <typename F>
__device__ __forceinline__ F warps_sum(F v, F (*sh)[32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  sh[warp][lane] = v;
  __syncthreads();
  F s = 0;
#pragma unroll 8
  for (int k = 0; k < kGnSumWarps; ++k) s += sh[k][lane];
  return s;
}

// mean and rstd of a sample's groups from the chunks' statistics
__global__ void __launch_bounds__(32 * kGnSumWarps) k_gn_join_stats(const Gn p, int blocks) {
  __shared__ double wide[kGnSumWarps][32];
  __shared__ float sh[kGnSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long n = blockIdx.x / unsigned(blocks);
  const int g = int(blockIdx.x - n * blocks) * 32 + lane;
  const bool on = g < p.groups;
  const float* part = p.part + (n * p.chunks * p.groups + (on ? g : 0)) * 3;
  const long long pitch = 3ll * p.groups;
  take_turn();
  const auto mean_of = [&](int c) { return double(part[c * pitch]) + double(part[c * pitch + 1]); };
  double s = 0.0;
#pragma unroll 4
  for (int c = warp; c < p.chunks; c += kGnSumWarps)
    s = __fma_rn(double(min(p.chunk_rows, p.rows - c * p.chunk_rows)), mean_of(c), s);
  const double mean = warps_sum(s, wide) / double(p.rows);
  float m2 = 0.f;
#pragma unroll 4
  for (int c = warp; c < p.chunks; c += kGnSumWarps) {
    const float have = float(min(p.chunk_rows, p.rows - c * p.chunk_rows)) * float(p.per);
    const float d = float(mean_of(c) - mean);
    m2 += fmaf(have * d, d, part[c * pitch + 2]);
  }
  m2 = warps_sum(m2, sh);
  if (on && warp == 0) {
    p.mean[n * p.groups + g] = float(mean);
    p.rstd[n * p.groups + g] = rsqrtf(m2 / (float(p.rows) * float(p.per)) + p.eps);
  }
}

// A sample's channel sums (sum e h, sum e) from those of its chunks
__global__ void __launch_bounds__(32 * kGnSumWarps) k_gn_join_grads(const Gn p, int blocks) {
  __shared__ float sh[kGnSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long n = blockIdx.x / unsigned(blocks);
  const int c = int(blockIdx.x - n * blocks) * 32 + lane;
  const bool on = c < p.channels;
  const float* part = p.part + n * p.chunks * 2 * p.channels + (on ? c : 0);
  take_turn();
  float s0 = 0.f, s1 = 0.f;
#pragma unroll 4
  for (int k = warp; k < p.chunks; k += kGnSumWarps) {
    s0 += part[2ll * k * p.channels];
    s1 += part[(2ll * k + 1) * p.channels];
  }
  s0 = warps_sum(s0, sh);
  s1 = warps_sum(s1, sh);
  if (on && warp == 0) {
    p.total[n * 2 * p.channels + c] = s0;
    p.total[(n * 2 + 1) * p.channels + c] = s1;
  }
}

// V parameters from channel c on; the type is looked at once.
template <int V>
__device__ __forceinline__ Vec<V> params_at(const void* q, int dtype, int c, float absent) {
  Vec<V> r = fill<V>(absent);
  if (!q) return r;
  if (dtype == EFCP_F32) {
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = static_cast<const float*>(q)[c + j];
  } else if (dtype == EFCP_BF16) {
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = to_f32(static_cast<const __nv_bfloat16*>(q)[c + j]);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = to_f32(static_cast<const __half*>(q)[c + j]);
  }
  return r;
}

// A thread's channel constants.
template <int V>
struct Lane {
  Vec<V> m, r, f, b;  // -mean, rstd, rstd weight, bias
  __device__ __forceinline__ void load(const Gn& p, const Item& it, int col) {
    const long long g = it.n * p.groups + it.g0;
    m = of_groups<V>(p.mean + g, col * V, p.per);
    r = of_groups<V>(p.rstd + g, col * V, p.per);
#pragma unroll
    for (int j = 0; j < V; ++j) m.v[j] = -m.v[j];
    f = r * params_at<V>(p.weight, p.param_dtype, it.c0 + col * V, 1.f);
    b = params_at<V>(p.bias, p.param_dtype, it.c0 + col * V, 0.f);
  }
};

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 6) k_gn_apply(const Gn p) {
  constexpr int U = kAhead<T, V>;
  const Item it = item_of<V>(p, blockIdx.x % unsigned(p.chunks), blockIdx.x / unsigned(p.chunks));
  take_turn();
  if (!it.on) return;
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  T* y = static_cast<T*>(p.y) + it.n * p.y_batch + it.c0;
  for (int c = it.tx; c < it.width / V; c += p.cols) {
    Lane<V> ln;
    ln.load(p, it, c);
    for (long long r = it.r0 + it.ty; r < it.r1; r += U * p.lanes_rows) {
      Pack<T, V> a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long rr = r + (long long)u * p.lanes_rows;
        if (rr < it.r1) a[u] = load_pack<T, V>(x + rr * p.x_row + (long long)c * V);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long rr = r + (long long)u * p.lanes_rows;
        if (rr < it.r1)
          *reinterpret_cast<Pack<T, V>*>(y + rr * p.y_row + (long long)c * V) =
              pack<T, V>(act_of<ACT>(fma(unpack(a[u]) + ln.m, ln.f, ln.b)));
      }
    }
  }
}

// Per channel and chunk of rows: sum e h, then sum e.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 4) k_gn_bwd_sums(const Gn p) {
  constexpr int U = kAhead<T, V>;
  extern __shared__ __align__(32) float sm[];
  float* val0 = sm;
  float* val1 = val0 + p.val_floats;
  const Item it = item_of<V>(p, blockIdx.x % unsigned(p.chunks), blockIdx.x / unsigned(p.chunks));
  take_turn();
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  const T* dy = static_cast<const T*>(p.dy) + it.n * p.dy_batch + it.c0;
  float* part = p.part + (it.n * p.chunks + it.chunk) * 2 * p.channels + it.c0;
  // the same rounds for every thread: there is a barrier inside
  for (int c0 = 0; c0 < it.width / V; c0 += p.cols) {
    const int c = c0 + it.tx;
    Vec<V> s0 = fill<V>(0.f), s1 = s0;
    if (it.on && c < it.width / V) {
      Lane<V> ln;
      ln.load(p, it, c);
      for (long long r = it.r0 + it.ty; r < it.r1; r += U * p.lanes_rows) {
        Pack<T, V> a[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long rr = r + (long long)u * p.lanes_rows;
          if (rr < it.r1) {
            a[u] = load_pack<T, V>(x + rr * p.x_row + (long long)c * V);
            d[u] = load_pack<T, V>(dy + rr * p.dy_row + (long long)c * V);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (r + (long long)u * p.lanes_rows < it.r1) {
            const Vec<V> q = unpack(a[u]) + ln.m;
            Vec<V> e = unpack(d[u]);
            if (ACT != EFCP_ACT_NONE) e = through_act<ACT>(e, fma(q, ln.f, ln.b));
            s0 = fma(e, q, s0);
            s1 = s1 + e;
          }
        }
      }
      s0 = s0 * ln.r;
    }
    sum_rows<V>(p, it, s0.v, val0);
    sum_rows<V>(p, it, s1.v, val1);
    __syncthreads();
    const int used = p.cols * V;
    for (int k = threadIdx.x; k < used && c0 * V + k < it.width; k += kGnThreads) {
      float t0 = 0.f, t1 = 0.f;
      for (int t = 0; t < p.val_rows; ++t) {
        t0 += val0[t * used + k];
        t1 += val1[t * used + k];
      }
      part[c0 * V + k] = t0;
      part[p.channels + c0 * V + k] = t1;
    }
    __syncthreads();
  }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 4) k_gn_bwd_apply(const Gn p) {
  constexpr int U = kAhead<T, V>;
  const Item it = item_of<V>(p, blockIdx.x % unsigned(p.chunks), blockIdx.x / unsigned(p.chunks));
  take_turn();
  // the groups' means of e w and of e w h
  extern __shared__ __align__(32) float joint[];
  {
    const float* total = p.total + it.n * 2 * p.channels + it.c0;
    const int lanes = 1 << p.lanes_log, lane = int(threadIdx.x) & (lanes - 1);
    for (int g0 = 0; g0 < it.ng; g0 += kGnThreads >> p.lanes_log) {
      const int g = g0 + (int(threadIdx.x) >> p.lanes_log);
      float sb = 0.f, sa = 0.f;
      if (g < it.ng) {
        for (int k = g * p.per + lane; k < (g + 1) * p.per; k += lanes) {
          const float w = weight_of(p, it.c0 + k);
          sb = fmaf(w, total[k], sb);
          sa = fmaf(w, total[p.channels + k], sa);
        }
      }
      sb = lanes_sum(sb, lanes);
      sa = lanes_sum(sa, lanes);
      if (g < it.ng && lane == 0) {
        joint[2 * g] = sa * p.inv_total;
        joint[2 * g + 1] = sb * p.inv_total;
      }
    }
  }
  __syncthreads();
  if (!it.on) return;
  const T* x = static_cast<const T*>(p.x) + it.n * p.x_batch + it.c0;
  const T* dy = static_cast<const T*>(p.dy) + it.n * p.dy_batch + it.c0;
  T* dx = static_cast<T*>(p.y) + it.n * p.y_batch + it.c0;
  for (int c = it.tx; c < it.width / V; c += p.cols) {
    Lane<V> ln;
    ln.load(p, it, c);
    Vec<V> qa, qb;
    GroupWalk walk(c * V, p.per);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      qa.v[j] = -joint[2 * walk.g];
      qb.v[j] = -joint[2 * walk.g + 1];
      walk.next(p.per);
    }
    qa = qa * ln.r;
    qb = qb * ln.r;
    for (long long r = it.r0 + it.ty; r < it.r1; r += U * p.lanes_rows) {
      Pack<T, V> a[U], d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long rr = r + (long long)u * p.lanes_rows;
        if (rr < it.r1) {
          a[u] = load_pack<T, V>(x + rr * p.x_row + (long long)c * V);
          d[u] = load_pack<T, V>(dy + rr * p.dy_row + (long long)c * V);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long rr = r + (long long)u * p.lanes_rows;
        if (rr < it.r1) {
          const Vec<V> q = unpack(a[u]) + ln.m;
          Vec<V> e = unpack(d[u]);
          if (ACT != EFCP_ACT_NONE) e = through_act<ACT>(e, fma(q, ln.f, ln.b));
          *reinterpret_cast<Pack<T, V>*>(dx + rr * p.y_row + (long long)c * V) =
              pack<T, V>(fma(q * ln.r, qb, fma(e, ln.f, qa)));
        }
      }
    }
  }
}

// dweight and dbias: column sums over `rows` rows of channel sums, in fp64 and a fixed order.  Eight
// channels per block, a sector of memory, so that few channels of many samples still occupy some SMs.
constexpr int kGnParamCols = 8;
__global__ void __launch_bounds__(32 * kGnSumWarps)
    k_gn_param_grads(const float* __restrict__ part, long long rows, int channels, int dtype,
                     void* dweight, void* dbias) {
  constexpr int kRows = 32 * kGnSumWarps / kGnParamCols;
  __shared__ double sh[2][kGnSumWarps][kGnParamCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = lane % kGnParamCols;
  const int c = int(blockIdx.x) * kGnParamCols + col;
  double s0 = 0.0, s1 = 0.0;
  take_turn();
  if (c < channels) {
#pragma unroll 4
    for (long long i = threadIdx.x / kGnParamCols; i < rows; i += kRows) {
      s0 += double(part[i * 2 * channels + c]);
      s1 += double(part[(i * 2 + 1) * channels + c]);
    }
  }
#pragma unroll
  for (int d = kGnParamCols; d < 32; d *= 2) {
    s0 += __shfl_xor_sync(~0u, s0, d);
    s1 += __shfl_xor_sync(~0u, s1, d);
  }
  if (lane < kGnParamCols) {
    sh[0][warp][col] = s0;
    sh[1][warp][col] = s1;
  }
  __syncthreads();
  if (warp < 2 && lane < kGnParamCols && c < channels) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kGnSumWarps; ++k) s += sh[warp][k][col];
    void* out = warp == 0 ? dweight : dbias;
    if (out) store_from_f32(out, dtype, c, float(s));
  }
}

// ------------------------------------------------------------------ launches
inline cudaError_t launch_params(const Gn& p, const float* sums, cudaStream_t st) {
  if (!p.dweight && !p.dbias) return cudaSuccess;
  const Shape s{unsigned((p.channels + kGnParamCols - 1) / kGnParamCols), 32 * kGnSumWarps, 0, 0};
  return launch(k_gn_param_grads, s, st, sums, p.n, p.channels, p.param_dtype, p.dweight, p.dbias);
}

template <typename T, int V, int ACT>
cudaError_t launch_act(const Gn& p, const GnLaunch& l) {
  if (l.resident) {
    const Shape s{l.blocks, kGnThreads, l.smem, unsigned(p.chunks)};
    if (!l.backward) return launch(k_gn_resident_fwd<T, V, ACT>, s, l.st, p);
    const cudaError_t e = launch(k_gn_resident_bwd<T, V, ACT>, s, l.st, p);
    return e != cudaSuccess ? e : launch_params(p, p.part, l.st);
  }
  const Shape sums{l.blocks, kGnThreads, size_t(gn_streamed_floats(p.val_floats, l.backward)) * 4, 0};
  const int joins = ((l.backward ? p.channels : p.groups) + 31) / 32;
  const Shape join{unsigned(p.n * joins), 32 * kGnSumWarps, 0, 0};
  const Shape apply{l.blocks, kGnThreads, l.backward ? size_t(p.tile_groups) * 8 : 0, 0};
  cudaError_t e;
  if (!l.backward) {
    e = launch(k_gn_stats<T, V>, sums, l.st, p);
    if (e == cudaSuccess) e = launch(k_gn_join_stats, join, l.st, p, joins);
    return e != cudaSuccess ? e : launch(k_gn_apply<T, V, ACT>, apply, l.st, p);
  }
  e = launch(k_gn_bwd_sums<T, V, ACT>, sums, l.st, p);
  if (e == cudaSuccess) e = launch(k_gn_join_grads, join, l.st, p, joins);
  if (e == cudaSuccess) e = launch(k_gn_bwd_apply<T, V, ACT>, apply, l.st, p);
  return e != cudaSuccess ? e : launch_params(p, p.total, l.st);
}

template <typename T, int V>
cudaError_t launch_vec(const Gn& p, const GnLaunch& l) {
  if (l.act == EFCP_ACT_NONE) return launch_act<T, V, EFCP_ACT_NONE>(p, l);
  if (l.act == EFCP_ACT_RELU) return launch_act<T, V, EFCP_ACT_RELU>(p, l);
  return launch_act<T, V, EFCP_ACT_SILU>(p, l);
}

}  // namespace
}  // namespace efcp
