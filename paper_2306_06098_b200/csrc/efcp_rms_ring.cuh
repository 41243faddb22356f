// RMS norm of rows that pass through shared memory (the plain kernels, and the formulas, are in efcp_rms.cuh).
//
// Bulk copies bring whole rows into shared memory while earlier ones are worked on, so that enough bytes are on
// their way without a register being held for them.  A group of warps asks for the next unit of a place when a barrier
// has told that all of them are done with the one there.
//
// A lane takes eight elements that lie together, on a multiple of eight of the logical order (row * d + column): the
// outputs and the groups of the dropout begin there.  Where rows do not begin so (ODD), a lane's eight may reach over the
// row's ends; an input that lies otherwise is read from shared memory in aligned pieces that are shifted into place; and
// a group's rows are a multiple of eight apart, so that its lanes keep their columns from row to row.  A place then holds
// whole pieces of 16 bytes, a row's neighbours in its ends, except before an input's first and behind its last element:
// those pieces' elements are copied one by one.
//
// The memory bounds rows that begin on 16 bytes without dropout, forward and backward: 16384 x 4096 bf16 with a residual
// 90 us (5.96 TB/s) and 108 us (4.97 TB/s); 16384 x 768, 16 us.  The rest waits on chains of instructions one behind the other, which
// the 16 warps on an SM that the registers allow do not hide (about half of the issue slots are used): dropout's ten rounds for eight
// elements (16384 x 768, 25 us, 53 % of them), the maxima and conversions of 8-bit outputs (8192 x 4096: 59 us, blocks of 128, 48 %),
// the shifts and the rows' ends of rows that begin anywhere (20000 x 1111 bf16: 53 us forward, 79 us backward; 117 and 153 with
// loads of single elements).
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_rms.h"
#include "efcp_rows.cuh"
#include "efcp_tc.cuh"

namespace efcp {
namespace {

constexpr int kRingFront = 48, kRingBack = 64;  // room around a place's rows (ODD): shifted pieces reach there

// (An input is read once; the cache is for the outputs, which are read next: 16384 x 768 bf16 forward 16.9 -> 15.7 us.)
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  uint64_t first_out;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(first_out));
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar), "l"(first_out)
      : "memory");
}

struct RingInput {
  const char* data;
  long long row;  // bytes between rows
};

// A group's view of its ring.
template <typename T, int INPUTS, bool ODD>
struct Ring {
  const Rms& p;
  const RmsRing& q;
  uint32_t data;  // of this group
  uint32_t bars;
  int* gave_up;
  long long first, step, units;  // units of the group: first, first + step, ...
  int group, warp, lane;
  RingInput in[INPUTS];
  int at = 0;  // place of the running unit, and the phase of its barrier
  uint32_t phase = 0;
  uint32_t plain = 0;  // see prepare()
  bool lost = false;   // a wait of this thread has run out
  long long asked = 0;  // (the asking thread) units asked for
  uint64_t limit = tc::kWaitNs;

  __device__ __forceinline__ uint32_t place(int s) const { return data + uint32_t(s * q.inputs * q.unit_bytes); }
  __device__ __forceinline__ void next() {
    if (++at == q.stages) {
      at = 0;
      phase ^= 1;
    }
  }
  // the warps of the group meet
  __device__ __forceinline__ void meet() const {
    if (p.warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(p.warps * 32) : "memory");
  }

  // Bytes lo .. hi of input i into shared memory (same place within 16 bytes).  With `issue` false: how many of them a
  // bulk copy takes, the others copied.
  __device__ __forceinline__ uint32_t pieces(int i, const char* lo, const char* hi, uint32_t to, uint32_t bar,
                                             bool issue) const {
    const char* const from = in[i].data;
    const char* const end = from + (p.rows - 1) * in[i].row + q.row_bytes;
    const char* a = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(lo) & ~uintptr_t(15));
    const char* b = reinterpret_cast<const char*>((reinterpret_cast<uintptr_t>(hi) + 15) & ~uintptr_t(15));
    if (a < from) a += 16;
    if (b > end) b -= 16;
    if (a >= b) a = b = hi;
    if (issue) {
      if (a < b) bulk_copy(to + uint32_t(a - lo), a, uint32_t(b - a), bar);  // (a - lo: -15 or more)
      return 0;
    }
    const auto one = [&](const char* x) {
      using Bits = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
      const Bits v = *reinterpret_cast<const Bits*>(x);
      if constexpr (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + uint32_t(x - lo)), "r"(v) : "memory");
      else asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + uint32_t(x - lo)), "h"(v) : "memory");
    };
    for (const char* x = lo; x < a; x += sizeof(T)) one(x);
    for (const char* x = b; x < hi; x += sizeof(T)) one(x);
    return uint32_t(b - a);
  }

  // ODD: what the copies of a unit bring in all, where one each does and a unit has others before and behind it; 0: not so.
  __device__ __forceinline__ uint32_t covered(uint32_t off, int i) const {
    return (off + uint32_t(in[i].row == q.row_bytes ? q.rows : 1) * q.row_bytes + 15) & ~15u;
  }
  __device__ __forceinline__ void prepare() {
    if constexpr (ODD) {
      plain = 0;
#pragma unroll
      for (int i = 0; i < INPUTS; ++i) {
        if (i >= q.inputs) break;
        if ((in[i].row != q.row_bytes && q.rows > 1) || in[i].row < 16) {
          plain = 0;
          return;
        }
        plain += covered(uint32_t(reinterpret_cast<uintptr_t>(in[i].data + first * q.rows * in[i].row) & 15), i);
      }
    }
  }

  // (one thread) unit u into place s.  Not when the wait for what is there has run out: its copies may still come, and the
  // barrier is not done with them.
  __device__ __forceinline__ void ask(long long u, int s) {
    if (u >= units || lost) return;
    ++asked;
    const int of_unit = q.rows * q.reps;
    const long long row = u * of_unit;
    const int rows = int(min((long long)of_unit, p.rows - row));
    const uint32_t bar = bars + 8 * s, to = place(s);
    if constexpr (!ODD) {
      tc::bar_expect(bar, uint32_t(rows * q.row_bytes * q.inputs));
#pragma unroll
      for (int i = 0; i < INPUTS; ++i) {
        if (i >= q.inputs) break;
        const char* from = in[i].data + row * in[i].row;
        if (in[i].row == q.row_bytes) bulk_copy(to + i * q.unit_bytes, from, uint32_t(rows * q.row_bytes), bar);
        else
          for (int r = 0; r < rows; ++r)
            bulk_copy(to + i * q.unit_bytes + r * q.row_bytes, from + r * in[i].row, uint32_t(q.row_bytes), bar);
      }
    } else if (u > 0 && u < units - 1 && plain) {
      tc::bar_expect(bar, plain);
#pragma unroll
      for (int i = 0; i < INPUTS; ++i) {
        if (i >= q.inputs) break;
        const char* lo = in[i].data + row * in[i].row;
        const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(lo) & 15);
        bulk_copy(to + i * q.unit_bytes + kRingFront, lo - off, covered(off, i), bar);
      }
    } else {
      const auto each = [&](bool issue) {
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < INPUTS; ++i) {
          if (i >= q.inputs) break;
          const bool whole = in[i].row == q.row_bytes;  // one row behind the other
          for (int r = 0; r < (whole ? 1 : rows); ++r) {
            const char* lo = in[i].data + (row + r) * in[i].row;
            bytes += pieces(i, lo, lo + (whole ? rows : 1) * q.row_bytes,
                            to + i * q.unit_bytes + kRingFront + r * q.pitch + uint32_t(reinterpret_cast<uintptr_t>(lo) & 15),
                            bar, issue);
          }
        }
        return bytes;
      };
      const uint32_t bytes = each(false);
      tc::bar_expect(bar, bytes);
      each(true);
    }
  }
  // Where column c of the lane's row in the group's units lies, in a place (the same for all of them).
  __device__ __forceinline__ uint32_t offset(int i, int sub, int c) const {
    const uint32_t col = uint32_t(c * int(sizeof(T)));
    if constexpr (!ODD) return i * q.unit_bytes + sub * q.row_bytes + col;
    const bool whole = in[i].row == q.row_bytes;
    const char* lo = in[i].data + (first * q.rows + (whole ? 0 : sub)) * in[i].row;
    return i * q.unit_bytes + kRingFront + uint32_t(reinterpret_cast<uintptr_t>(lo) & 15) +
           sub * (whole ? q.row_bytes : q.pitch) + col;
  }
  // The running unit has arrived.  When the limit passes the work goes on with whatever lies there (the warps of a
  // group keep meeting) without further waits, and the status tells.
  __device__ __forceinline__ void await() {
    if (!lost) lost = !tc::bar_wait(bars + 8 * at, phase, gave_up, limit);
  }
  // Nothing may land in shared memory that the block has left.
  __device__ __forceinline__ void end() const {
    if (!*(volatile int*)gave_up) return;
    for (long long n = asked < q.stages ? 0 : asked - q.stages; n < asked; ++n)
      (void)tc::bar_wait(bars + 8 * int(n % q.stages), uint32_t(n / q.stages) & 1, gave_up, tc::kDrainNs);
  }
};

// (all threads) Tells when a wait of any group has run out.  Groups come here at different times, so the block meets first.
__device__ __forceinline__ void ring_tell(int* status, volatile int* gave_up) {
  __syncthreads();
  if (threadIdx.x == 0 && *gave_up) atomicExch(status, EFCP_ETIMEOUT);
}

// Barriers, and the group that a warp belongs to.  (Up to 8 groups of up to 4 places.)
template <typename T, int INPUTS, bool ODD>
__device__ __forceinline__ Ring<T, INPUTS, ODD> ring_begin(const Rms& p, const RmsRing& q, unsigned char* smem,
                                                           int* gave_up) {
  const int warp = threadIdx.x >> 5;
  const uint32_t bars = tc::smem_of(smem);
  if (threadIdx.x == 0) {
    *gave_up = 0;
    for (int i = 0; i < p.groups * q.stages; ++i) tc::bar_init(bars + 8 * i, 1);
    tc::bar_init_fence();
  }
  const int g = warp / p.warps;
  return Ring<T, INPUTS, ODD>{p, q, tc::smem_of(smem) + q.data_at + uint32_t(g * q.stages * q.inputs * q.unit_bytes),
                              bars + 8 * g * q.stages, gave_up,
                              (long long)blockIdx.x * p.groups + g, (long long)gridDim.x * p.groups,
                              (p.rows + q.rows * q.reps - 1) / (q.rows * q.reps), g, warp - g * p.warps,
                              int(threadIdx.x) & 31, {}};
}

// A lane's columns: c, c + step, ... of its row in each unit.
struct RingCols {
  int sub, c, step;
  bool lead;        // the row's first lane
  uint32_t weight;  // where the weight of its first eight lies, and how far apart the next are
  uint32_t weight_step;
};

template <int K, bool ODD, typename R>
__device__ __forceinline__ RingCols ring_cols(const R& r, unsigned char* smem) {
  const Rms& p = r.p;
  const RmsRing& q = r.q;
  RingCols a;
  a.sub = r.lane / q.lanes;
  const int l = r.lane - a.sub * q.lanes;
  a.step = p.warps * kChunk;
  a.c = l * 8 + r.warp * kChunk;
  a.lead = l == 0 && r.warp == 0;
  float* weight = reinterpret_cast<float*>(smem + q.weight_at);
  if constexpr (ODD) {
    a.c -= int(((r.first * q.rows + a.sub) * p.d) & 7);
    // each lane's own, as it reads them
    float* mine = weight + (int(threadIdx.x >> 5) * K * 32 + r.lane) * 8;
    const auto copy = [&](const auto* w) {
#pragma unroll 1
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = a.c + k * a.step + j;
          mine[k * kChunk + j] = c >= 0 && c < p.d ? to_f32(w[c]) : 0.f;
        }
    };
    if (p.weight) {
      if (p.param_dtype == EFCP_F32) copy(static_cast<const float*>(p.weight));
      else if (p.param_dtype == EFCP_BF16) copy(static_cast<const __nv_bfloat16*>(p.weight));
      else copy(static_cast<const __half*>(p.weight));
    }
    a.weight = tc::smem_of(mine);
    a.weight_step = kChunk * 4;
  } else {
    if (p.weight)
      for (int c = threadIdx.x; c < p.d; c += blockDim.x) weight[c] = load_as_f32(p.weight, p.param_dtype, c);
    a.weight = tc::smem_of(weight) + a.c * 4;
    a.weight_step = a.step * 4;
  }
  return a;
}

// Eight elements as they lie in memory.
template <typename T>
struct Eight {
  static constexpr int kWords = int(sizeof(T)) * 2;
  uint32_t w[kWords];

  static __device__ __forceinline__ void four(uint32_t* to, uint32_t at) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(to[0]), "=r"(to[1]), "=r"(to[2]), "=r"(to[3])
                 : "r"(at)
                 : "memory");
  }
  // (SHIFT: `at` need not be a multiple of 16)
  template <bool SHIFT>
  __device__ __forceinline__ void load_shared(uint32_t at) {
    if constexpr (!SHIFT) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) four(w + i, at + 4 * i);
    } else {
      const uint32_t shift = at & 15, from = at & ~15u;
      uint32_t a[kWords + 4];
#pragma unroll
      for (int i = 0; i < kWords; i += 4) four(a + i, from + 4 * i);
      if (shift) {
        four(a + kWords, from + 4 * kWords);
        if (shift & 8) {
#pragma unroll
          for (int i = 0; i < kWords + 2; ++i) a[i] = a[i + 2];
        }
        if (shift & 4) {
#pragma unroll
          for (int i = 0; i < kWords + 1; ++i) a[i] = a[i + 1];
        }
        if (sizeof(T) == 2 && (shift & 2)) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) a[i] = __funnelshift_r(a[i], a[i + 1], 16);
        }
      }
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = a[i];
    }
  }
  __device__ __forceinline__ void load(const T* from) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(from) + i);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void store(T* to) const {
#pragma unroll
    for (int i = 0; i < kWords; i += 4)
      *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(to) + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  }
  // columns c .. c + 7 of a row of d  (EDGES: some of them may lie outside)
  template <bool EDGES>
  __device__ __forceinline__ void store(T* row, int c, int d) const {
    if (!EDGES || (c >= 0 && c + 8 <= d)) {
      store(row + c);
    } else {
      using Bits = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j >= 0 && c + j < d)
          reinterpret_cast<Bits*>(row)[c + j] = sizeof(T) == 4 ? Bits(w[j % kWords]) : Bits(w[j / 2] >> (16 * (j & 1)));
    }
  }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        v[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
      } else {
        const __half2 h = reinterpret_cast<const __half2&>(w[i]);
        v[i] = __half22float2(h);
      }
    }
  }
  __device__ __forceinline__ void set(const float2 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        w[2 * i] = __float_as_uint(v[i].x);
        w[2 * i + 1] = __float_as_uint(v[i].y);
      } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        const __nv_bfloat162 h = __float22bfloat162_rn(v[i]);
        w[i] = reinterpret_cast<const uint32_t&>(h);
      } else {
        const __half2 h = __float22half2_rn(v[i]);
        w[i] = reinterpret_cast<const uint32_t&>(h);
      }
    }
  }
};

// zeros for what lies outside of a row of d
template <bool EDGES>
__device__ __forceinline__ void only_row(float2 (&v)[4], int c, int d) {
  if (EDGES && (c < 0 || c + 8 > d)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (unsigned(c + 2 * i) >= unsigned(d)) v[i].x = 0.f;
      if (unsigned(c + 2 * i + 1) >= unsigned(d)) v[i].y = 0.f;
    }
  }
}

__device__ __forceinline__ void drop_pairs(float2 (&v)[4], unsigned long long group, const DropKey& key,
                                           const Drop& drop) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { w[2 * i] = v[i].x; w[2 * i + 1] = v[i].y; }
  drop_group(w, group, key, drop.threshold, drop.scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float2(w[2 * i], w[2 * i + 1]);
}

// Sum (or maximum of magnitudes) over the lanes and warps that share a row; `slot` tells the exchanges of one row apart,
// and a barrier lies between two uses of the same slot.
template <bool MAX, typename R>
__device__ __forceinline__ float ring_join(const R& r, float v, int slot) {
  __shared__ alignas(16) float part[4][8][8];
  const auto join = [](float a, float b) {
    if constexpr (MAX) return larger(a, b);
    else return a + b;
  };
  if (r.q.lanes == 32) {
    if constexpr (MAX) {
      v = lanes_max(v, 32);
    } else {
#pragma unroll
      for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    }
  } else {
    for (int o = r.q.lanes / 2; o; o >>= 1) v = join(v, __shfl_xor_sync(kAll, v, o));
  }
  if (r.p.warps == 1) {
    __syncwarp();
    return v;
  }
  float* mine = part[slot][r.group];
  if (r.lane == 0) mine[r.warp] = v;
  if (r.lane == 1 && r.warp == 0)
    for (int i = r.p.warps; i < 8; ++i) mine[i] = 0.f;
  r.meet();
  const float4 a = *reinterpret_cast<const float4*>(mine), b = *reinterpret_cast<const float4*>(mine + 4);
  return join(join(join(a.x, a.y), join(a.z, a.w)), join(join(b.x, b.y), join(b.z, b.w)));
}

__device__ __forceinline__ float max_nan3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// The largest magnitude, NaN where there is one.
__device__ __forceinline__ float most_of(const float2 (&v)[4]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max_nan3(m, fabsf(v[i].x), fabsf(v[i].y));
  return m;
}

// K: chunks of a warp; h stays in registers.  SUM: h may be other than x; DROP: with dropout.
template <typename T, int K, int QUANT, bool SUM, bool DROP, bool ODD>
__global__ void __launch_bounds__(256, 2) k_rms_forward_ring(const Rms p, const RmsRing q) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int gave_up;
  constexpr int kInputs = SUM ? 2 : 1;
  auto r = ring_begin<T, kInputs, ODD>(p, q, smem, &gave_up);
  r.in[0] = {static_cast<const char*>(p.x), p.x_row * (long long)sizeof(T)};
  if constexpr (SUM) r.in[1] = {static_cast<const char*>(p.residual), p.residual_row * (long long)sizeof(T)};
  r.prepare();
  take_turn();
  __syncthreads();
  const bool asks = r.warp == 0 && r.lane == 0;
  if (asks)
    for (int n = 0; n < q.stages; ++n) r.ask(r.first + n * r.step, n);
  const RingCols me = ring_cols<K, ODD>(r, smem);
  __syncthreads();
  DropKey key{};
  if constexpr (DROP) key = drop_key(p.drop);
  const bool two = SUM && p.residual, kept = SUM && p.h;
  const uint32_t x0 = r.offset(0, me.sub, me.c), res0 = two ? r.offset(1, me.sub, me.c) : 0;
  unsigned odd = 0;
  for (long long u = r.first; u < r.units; u += r.step) {
    r.await();
    for (int rep = 0; rep < q.reps; ++rep, odd ^= 1) {
      const long long row = (u * q.reps + rep) * q.rows + me.sub;
      const bool on = row < p.rows && me.sub < q.rows;
      const uint32_t skip = r.place(r.at) + uint32_t(rep * q.rows * q.row_bytes), x = skip + x0, res = skip + res0;
      const long long at = row * p.d;
      Eight<T> h[K];
      float2 sq = both(0.f);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = me.c + k * me.step;
        if (!on || c >= p.d) continue;
        h[k].template load_shared<ODD>(x + k * me.step * sizeof(T));
        float2 v[4];
        h[k].get(v);
        if constexpr (SUM) {
          if constexpr (DROP) drop_pairs(v, (unsigned long long)(at + c) >> 3, key, p.drop);
          if (two) {
            Eight<T> a;
            a.template load_shared<ODD>(res + k * me.step * sizeof(T));
            float2 w[4];
            a.get(w);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = add2(v[i], w[i]);
          }
          if (kept) {
            h[k].set(v);
            h[k].template store<ODD>(static_cast<T*>(p.h) + at, c, p.d);
            h[k].get(v);
          }
        }
        only_row<ODD>(v, c, p.d);
        float2 t = mul2(v[0], v[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) t = fma2(v[i], v[i], t);
        sq = fma2(t, both(p.inv_d), sq);
      }
      const float rstd = rsqrtf(ring_join<false>(r, sq.x + sq.y, int(odd)) + p.eps);
      // every warp of the group is done with this place
      if (asks && rep == q.reps - 1) r.ask(u + q.stages * r.step, r.at);
      if (on && me.lead && p.rstd) p.rstd[row] = rstd;
      const auto norm8 = [&](int k, float2(&v)[4]) {
        h[k].get(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], both(rstd));
        if (p.weight) {
          Eight<float> w;
          w.template load_shared<false>(me.weight + k * me.weight_step);
          float2 f[4];
          w.get(f);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f[i]);
        }
      };
      if constexpr (QUANT == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int c = me.c + k * me.step;
          if (!on || c >= p.d) continue;
          float2 v[4];
          norm8(k, v);
          Eight<T> y;
          y.set(v);
          y.template store<ODD>(static_cast<T*>(p.y) + at, c, p.d);
        }
      } else {
        float* scales = p.scales + row * p.blocks;
        unsigned char* out = static_cast<unsigned char*>(p.y) + at;
        float one = 1.f, inv = 1.f;
        if (p.block == 0) {
          float top = 0.f;
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const int c = me.c + k * me.step;
            if (!on || c >= p.d) continue;
            float2 z[4];
            norm8(k, z);
            only_row<ODD>(z, c, p.d);
            top = larger(top, most_of(z));
          }
          one = scale_of(ring_join<true>(r, top, 2 + int(odd)), p.most);
          inv = inverse_of(one);
          if (on && me.lead) scales[0] = one;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int c = me.c + k * me.step;
          const bool here = on && c < p.d;
          float2 z[4] = {};
          if (here) norm8(k, z);
          if (!ODD && p.block) {  // (all lanes: the maximum of a block is exchanged between them)
            float top = most_of(z);
            const int lanes = min(p.block / 8, q.lanes);
            if (lanes > 1) top = larger(top, __shfl_xor_sync(kAll, top, 1));
            if (lanes > 2) top = larger(top, __shfl_xor_sync(kAll, top, 2));
            if (lanes > 4) top = larger(top, __shfl_xor_sync(kAll, top, 4));
            if (lanes > 8) top = larger(top, __shfl_xor_sync(kAll, top, 8));
            one = scale_of(top, p.most);
            inv = inverse_of(one);
            if (here && (c & (p.block - 1)) == 0) scales[c >> p.block_shift] = one;
          }
          if (!here) continue;
          const uint2 o = quantized8<QUANT == 1>(z, one, inv);
          if (!ODD || (c >= 0 && c + 8 <= p.d)) {
            *reinterpret_cast<uint2*>(out + c) = o;
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (c + j >= 0 && c + j < p.d) out[c + j] = (unsigned char)((j < 4 ? o.x : o.y) >> (8 * (j & 3)));
          }
        }
      }
    }
    r.next();
  }
  if (asks) r.end();
  ring_tell(p.status, &gave_up);
}

// K: chunks of a warp; it holds their sums of the weight's gradient in registers.
template <typename T, int K, bool DROP, bool ODD>
__global__ void __launch_bounds__(256, 2) k_rms_backward_ring(const Rms p, const RmsRing q) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int gave_up;
  auto r = ring_begin<T, 3, ODD>(p, q, smem, &gave_up);
  r.in[0] = {static_cast<const char*>(p.dy), p.dy_row * (long long)sizeof(T)};
  r.in[1] = {static_cast<const char*>(p.x), p.x_row * (long long)sizeof(T)};
  r.in[2] = {static_cast<const char*>(p.dh), p.dh_row * (long long)sizeof(T)};
  r.prepare();
  take_turn();
  __syncthreads();
  const bool asks = r.warp == 0 && r.lane == 0;
  if (asks)
    for (int n = 0; n < q.stages; ++n) r.ask(r.first + n * r.step, n);
  const RingCols me = ring_cols<K, ODD>(r, smem);
  __syncthreads();
  DropKey key{};
  if constexpr (DROP) key = drop_key(p.drop);
  const uint32_t dy0 = r.offset(0, me.sub, me.c), h0 = r.offset(1, me.sub, me.c),
                 dh0 = p.dh ? r.offset(2, me.sub, me.c) : 0;
  float2 dw[K][4];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[k][i] = both(0.f);
  const auto rstd_of = [&](long long unit, int rep) {
    const long long row = (unit * q.reps + rep) * q.rows + me.sub;
    return row < p.rows ? p.rstd[row] : 0.f;
  };
  const auto weight8 = [&](int k, float2(&w)[4]) {
    Eight<float> a;
    a.template load_shared<false>(me.weight + k * me.weight_step);
    a.get(w);
  };
  unsigned odd = 0;
  float next = rstd_of(r.first, 0);
  for (long long u = r.first; u < r.units; u += r.step) {
    r.await();
    for (int rep = 0; rep < q.reps; ++rep, odd ^= 1) {
      const long long row = (u * q.reps + rep) * q.rows + me.sub;
      const bool on = row < p.rows && me.sub < q.rows;
      const uint32_t skip = r.place(r.at) + uint32_t(rep * q.rows * q.row_bytes), dy = skip + dy0, h = skip + h0,
                     dh = skip + dh0;
      const long long at = row * p.d;
      const float rs = next;
      next = rep + 1 < q.reps ? rstd_of(u, rep + 1) : rstd_of(u + r.step, 0);
      Eight<T> a8[K], b8[K], e8[K];
      float2 sum = both(0.f);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = me.c + k * me.step;
        if (!on || c >= p.d) continue;
        a8[k].template load_shared<ODD>(dy + k * me.step * sizeof(T));
        b8[k].template load_shared<ODD>(h + k * me.step * sizeof(T));
        if (p.dh) e8[k].template load_shared<ODD>(dh + k * me.step * sizeof(T));
        float2 a[4], b[4];
        if constexpr (ODD) {
          if (c < 0 || c + 8 > p.d) {
            a8[k].get(a);
            only_row<ODD>(a, c, p.d);
            a8[k].set(a);
            b8[k].get(b);
            only_row<ODD>(b, c, p.d);
            b8[k].set(b);
          }
        }
        a8[k].get(a);
        b8[k].get(b);
        if (p.weight) {
          float2 w[4];
          weight8(k, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = mul2(a[i], w[i]);
        }
        float2 t = mul2(a[0], b[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) t = fma2(a[i], b[i], t);
        sum = add2(sum, t);
      }
      const float m = -ring_join<false>(r, sum.x + sum.y, int(odd)) * p.inv_d * rs * rs;
      // every warp of the group is done with this place
      if (asks && rep == q.reps - 1) r.ask(u + q.stages * r.step, r.at);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = me.c + k * me.step;
        if (!on || c >= p.d) continue;
        float2 a[4], b[4];
        a8[k].get(a);
        b8[k].get(b);
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[k][i] = fma2(a[i], mul2(b[i], both(rs)), dw[k][i]);
        if (p.weight) {
          float2 w[4];
          weight8(k, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = mul2(a[i], w[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = mul2(fma2(b[i], both(m), a[i]), both(rs));
        if (p.dh) {
          float2 e[4];
          e8[k].get(e);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = add2(a[i], e[i]);
        }
        Eight<T> out;
        if (p.dresidual) {
          out.set(a);
          out.template store<ODD>(static_cast<T*>(p.dresidual) + at, c, p.d);
        }
        if (p.dx) {
          if constexpr (DROP) drop_pairs(a, (unsigned long long)(at + c) >> 3, key, p.drop);
          out.set(a);
          out.template store<ODD>(static_cast<T*>(p.dx) + at, c, p.d);
        }
      }
    }
    r.next();
  }
  if (asks) r.end();
  ring_tell(p.status, &gave_up);
  if (p.part) {
    // The rows of a block's warps, each in its place of shared memory (the rings are done with), are added up in order.
    float* sums = reinterpret_cast<float*>(smem + q.data_at);
    float* const out = p.part + (long long)blockIdx.x * p.d;
    const bool alone = p.groups * q.rows == 1;
    float* mine = alone ? out : sums + (r.group * q.rows + me.sub) * p.d;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = me.c + k * me.step;
      if (c >= p.d) continue;
      Eight<float> a;
      a.set(dw[k]);
      if constexpr (!ODD) {
        a.store(mine + c);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (unsigned(c + j) < unsigned(p.d)) mine[c + j] = __uint_as_float(a.w[j]);
      }
    }
    if (alone) return;
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
      float v = sums[c];
      for (int i = 1; i < p.groups * q.rows; ++i) v += sums[i * p.d + c];
      out[c] = v;
    }
  }
}

template <typename T, int K, bool ODD>
cudaError_t rms_launch_ring_k(const Rms& p, const RmsLaunch& l) {
  const Shape s{l.blocks, unsigned(p.groups * p.warps * 32), l.smem, 0};
  const bool sum = p.h || ODD, drop = p.drop.threshold;
  switch (l.op) {
    case kRmsE4M3:
      return sum ? launch(k_rms_forward_ring<T, K, 1, true, false, ODD>, s, l.st, p, l.ring)
                 : launch(k_rms_forward_ring<T, K, 1, ODD, false, ODD>, s, l.st, p, l.ring);
    case kRmsInt8:
      return sum ? launch(k_rms_forward_ring<T, K, 2, true, false, ODD>, s, l.st, p, l.ring)
                 : launch(k_rms_forward_ring<T, K, 2, ODD, false, ODD>, s, l.st, p, l.ring);
    case kRmsForward:
      return drop  ? launch(k_rms_forward_ring<T, K, 0, true, true, ODD>, s, l.st, p, l.ring)
             : sum ? launch(k_rms_forward_ring<T, K, 0, true, false, ODD>, s, l.st, p, l.ring)
                   : launch(k_rms_forward_ring<T, K, 0, ODD, false, ODD>, s, l.st, p, l.ring);
    default:
      return drop ? launch(k_rms_backward_ring<T, K, true, ODD>, s, l.st, p, l.ring)
                  : launch(k_rms_backward_ring<T, K, false, ODD>, s, l.st, p, l.ring);
  }
}

template <typename T, bool ODD>
cudaError_t rms_launch_ring(const Rms& p, const RmsLaunch& l) {
  return l.kept == 1   ? rms_launch_ring_k<T, 1, ODD>(p, l)
         : l.kept == 2 ? rms_launch_ring_k<T, 2, ODD>(p, l)
                       : rms_launch_ring_k<T, 4, ODD>(p, l);
}

}  // namespace
}  // namespace efcp
