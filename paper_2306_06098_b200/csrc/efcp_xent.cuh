// Softmax cross entropy of a linear layer over a vocabulary (the formulas stand in include/efcp.h), in products of
// tiles on the fifth-generation tensor cores.  The logits never reach memory: a tile of them is turned into the rows'
// largest value and sum of exponentials, and in the backward pass, computed once more for a piece of the vocabulary
// at a time, into their gradient, which the two products behind it read.  One launch holds both products of a piece
// and the logits of the next one, so that few tiles are left over at its end.
//
// A pair of blocks on neighbouring SMs works on a tile of 256 x 256: each block holds 128 rows of it in its tensor
// memory, and loads its rows of one operand and half of the other, which the instructions of the pair share.  In each block
// a warp copies operands into a ring in shared memory, and eight warps work on one of two accumulators while the
// tensor cores fill the other; a warp of the first block issues the products.  Every wait is bounded; when one runs out
// the blocks end, and the status tells of it.
//
// The tensor cores cut what they add up to fp32 instead of rounding it, 16 products at a time.  An accumulator holds no more products
// than may be added up so (part_of), and the parts are added up in registers, rounded.
//
// With 16-bit operands the logits' gradient is rounded to their type, but for the entries of the targets, by far the largest: without
// what that rounding leaves of them the gradients are 0.0017 off (2-norm, 2458 x 256 x 30522 bf16), with it below 0.0001, where the
// results' own rounding is 0.0017.  The gradient of H gets it in k_xent_finish, the gradient of W in steps of its own, with the tokens
// whose targets are near (XentGemm::bounds).
//
// fp32 values are held as three bfloat16 ones (8 bits of the significand each), of whose nine products the six
// largest are added up, the small ones first.  What is left out is below 2^-22 of the sum of the products' magnitudes: two products
// of at most 2^-24 each, and a smaller one.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "efcp.h"
#include "efcp_launch.cuh"
#include "efcp_num.cuh"
#include "efcp_rows.cuh"
#include "efcp_tc.cuh"
#include "efcp_xent.h"

namespace efcp {
namespace {

constexpr int kStages = 6;
constexpr int kOutWarps = 8, kXentThreads = (kOutWarps + 4) * 32;
constexpr int kBlockRows = kXentRows / 2;       // of a tile, held by a block
constexpr uint32_t kBoxBytes = 64 * 128;        // 64 rows of 64 elements
constexpr uint32_t kABytes = kBlockRows / 64 * kBoxBytes, kBBytes = kXentCols / 128 * kBoxBytes;
constexpr uint32_t kStageBytes = kABytes + kBBytes;
constexpr uint32_t kOutBytes = 32 * 128;        // a warp's box of results
constexpr size_t kXentSmem = kStages * kStageBytes + kOutWarps * kOutBytes + 1024;
constexpr int kRestWarps = 3;                   // see load_rests
constexpr int kSquare = 8;                      // rows of tiles that pairs work on side by side

template <typename T>
using Operand = std::conditional_t<std::is_same_v<T, __half>, __half, __nv_bfloat16>;

__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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

enum XentKind { kHidden, kWeight, kLogits };

// Steps of an accumulator, from step i of a tile on.  What the tensor cores cut is of the size of the running sum: of fp32 operands the
// products of the largest parts come last, and the others may be added up longer.  (Mean error of lse, 1003 x 509 x 10007 fp32:
// -0.9e-6; with eight steps for all -3.4e-6, and no faster.  2048 x 4096 x 8000 fp16: four steps -2.1e-6, eight -4.0e-6.)  The logits
// are the same in both directions, so that a row's probabilities add up to one (fp16, 4096 products of one sign: 6e-4 short of it
// with one accumulator); the products with G, whose results are 16 bits, may be longer (131072 tokens of one sign, fp16: 1e-5 off
// with 64 steps, 9e-4 with one accumulator; that is 6 % on 8192 x 4096 x 64000).
template <bool F32>
__device__ __forceinline__ int part_of(XentKind kind, int i, int depth, int steps) {
  if constexpr (F32) {
    const int small = 5 * depth;
    return i < small ? min(32, small - i) : min(2, steps - i);
  } else {
    return min(kind == kLogits ? 4 : 64, steps - i);
  }
}

struct XentTile {
  XentKind kind;
  int m0, n0;     // rows and columns of the result
  int cols;       // width of the tile
  int k0, depth;  // first step along the sum, and steps
  int rest0, rests;  // the same of the steps that bring what the rounding of G left (weight)
  int part;       // of the sum over the piece (hidden); tile of the columns (logits)
};

// The tiles of a launch, eight rows of tiles by as many columns as there are pairs at a time for the products of G, which
// does not stay in the cache (8192 x 8192 bf16: read twice instead of seven times); all rows first for the logits: H does.
struct XentWork {
  int row_tiles, weight_rows, splits, steps, token_steps;
  int shift, piece, v0, next_v0, col_tiles;  // pieces: the one that hidden and weight read, the one that logits writes
  int rows, next_cols;                       // of them: rows of W, columns
  long long hidden, weight, all;             // tiles of hidden; and of weight; and of logits
  bool six;                                  // products for each step

  __device__ __forceinline__ XentWork(const XentGemm& p, int count, int pairs, bool backward, bool six_) {
    six = six_;
    row_tiles = (count + kXentRows - 1) / kXentRows;
    shift = backward ? xent_shift(row_tiles, p.tiles, p.shifts) : 0;
    piece = p.piece << shift;
    col_tiles = p.col_tiles << shift;
    // (what begins behind the vocabulary is not worked on)
    const long long begin = backward ? (p.turn - 1ll) * piece : 0, next = backward ? (long long)p.turn * piece : 0;
    const bool products = begin >= 0 && begin < p.vocab && backward, logits = next < p.vocab;
    v0 = products ? int(begin) : 0;
    next_v0 = logits ? int(next) : 0;
    rows = min(piece, p.vocab - v0);
    next_cols = min(piece, p.vocab - next_v0);
    // (the last piece's tiles end with the vocabulary: pieces are whole tiles, or there is one)
    if (backward) col_tiles = min(col_tiles, (next_cols + p.col_tile - 1) / p.col_tile);
    weight_rows = (rows + kXentRows - 1) / kXentRows;
    steps = (rows + kXentDepth - 1) / kXentDepth;
    token_steps = (count + kXentDepth - 1) / kXentDepth;
    splits = xent_splits(row_tiles, p.d_tiles, piece, pairs, six);
    hidden = products && p.hidden ? (long long)row_tiles * p.d_tiles * splits : 0;
    weight = hidden + (products && p.weight ? (long long)weight_rows * p.d_tiles : 0);
    all = weight + (logits ? (long long)row_tiles * col_tiles : 0);
  }
  static __device__ __forceinline__ int2 square(int t, int rows, int cols) {
    const int g = t / (kSquare * cols), first = g * kSquare, here = min(kSquare, rows - first);
    t -= first * cols;
    const int c = t / here;
    return make_int2(first + t - c * here, c);
  }
  __device__ __forceinline__ XentTile tile(const XentGemm& p, long long t) const {
    XentTile r;
    r.rest0 = r.rests = 0;
    if (t < hidden) {
      const int2 mn = square(int(t), row_tiles, p.d_tiles * splits);
      const int n = mn.y / splits;
      r.kind = kHidden;
      r.m0 = mn.x * kXentRows;
      r.n0 = n * p.d_tile;
      r.cols = p.d_tile;
      r.part = mn.y - n * splits;
      const int per = (steps + splits - 1) / splits;
      r.k0 = min(steps, r.part * per);
      r.depth = min(per, steps - r.k0);
    } else if (t < weight) {
      const int2 mn = square(int(t - hidden), weight_rows, p.d_tiles);
      r.kind = kWeight;
      r.m0 = mn.x * kXentRows;
      r.n0 = mn.y * p.d_tile;
      r.cols = p.d_tile;
      r.part = r.k0 = 0;
      r.depth = token_steps;
      if (!six) {
        const int bucket = (v0 + r.m0) / kXentRows >> p.wide, first = p.bounds[bucket], last = p.bounds[bucket + 1];
        r.rest0 = first / kXentDepth;
        r.rests = last > first ? (last - 1) / kXentDepth - r.rest0 + 1 : 0;
      }
    } else {
      t -= weight;
      const int c = int(t / row_tiles);
      r.kind = kLogits;
      r.m0 = int(t - (long long)c * row_tiles) * kXentRows;
      r.n0 = c * p.col_tile;
      r.cols = p.col_tile;
      r.part = c;
      r.k0 = 0;
      r.depth = (p.d + kXentDepth - 1) / kXentDepth;
    }
    return r;
  }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 2^(v log2(e) - base), two at a time
__device__ __forceinline__ float2 exp_pair(float a, float b, float base) {
  const float2 x = fma2(make_float2(a, b), both(kLog2e), both(-base));
  return make_float2(pow2(x.x), pow2(x.y));
}

// A row's lse, for its probabilities: e^(v - lse) = 2^(v log2(e) - base) scale.  (lse times log2(e) is rounded to its own size, by much
// more than a probability near 1 may be off; what that leaves is in the scale, which is a little off 1.)
struct RowLse {
  float base = 0.f, scale = 1.f;
  __device__ __forceinline__ void set(float lse) {
    base = lse * kLog2e;
    const float x = -0.69314718f * fmaf(lse, kLog2e, -base);  // (below 2^-24 of lse: two terms of the exponential)
    scale = fmaf(fmaf(0.5f, x, 1.f), x, 1.f);
  }
};

// What becomes of 32 columns of a row of logits, forward: their largest value (times log2(e)) and the sum of
// exponentials relative to it are joined to the row's.
struct RowStats {
  float top = -INFINITY, total = 0.f;
  __device__ __forceinline__ void add(const XentGemm& p, int row, int target, int col, float (&v)[32]) {
    const int valid = p.vocab - col;
    if (valid <= 0) return;
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
    float m = fmaxf(v[0], v[1]), n = fmaxf(v[2], v[3]);
#pragma unroll
    for (int i = 4; i < 32; i += 4) {
      m = max3(m, v[i], v[i + 1]);
      n = max3(n, v[i + 2], v[i + 3]);
    }
    m = fmaxf(top, fmaxf(m, n) * kLog2e);
    const float base = m == -INFINITY ? 0.f : m;
    total *= pow2(top - base);
    top = m;
    float2 s = both(0.f), t = both(0.f);
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      s = add2(s, exp_pair(v[i], v[i + 1], base));
      t = add2(t, exp_pair(v[i + 2], v[i + 3], base));
    }
    s = add2(s, t);
    total += s.x + s.y;
  }
};

// Results leave through shared memory, 32 rows of 128 (or 64) bytes at a time for each warp, swizzled, so that its
// lanes, a row each, write to different banks.
template <typename O, int BYTES = 128>
struct OutBox {
  uint32_t at;  // of the warp
  int lane;
  // 16-byte pieces `first`, ... of the lane's row
  __device__ __forceinline__ void put(int first, const float (&v)[32]) const {
    constexpr int kPer = 16 / sizeof(O);
#pragma unroll
    for (int k = 0; k < 32 / kPer; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(O) == 4) {
          w[i] = __float_as_uint(v[k * 4 + i]);
        } else {
          const float2 x = make_float2(v[k * 8 + 2 * i], v[k * 8 + 2 * i + 1]);
          if constexpr (std::is_same_v<O, __half>) {
            const __half2 h = __float22half2_rn(x);
            w[i] = reinterpret_cast<const uint32_t&>(h);
          } else {
            const __nv_bfloat162 h = __float22bfloat162_rn(x);
            w[i] = reinterpret_cast<const uint32_t&>(h);
          }
        }
      }
      const int swizzle = BYTES == 128 ? lane & 7 : (lane >> 1) & 3;
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(
                       at + lane * BYTES + (((first + k) ^ swizzle) << 4)),
                   "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                   : "memory");
    }
  }
  // (fp32) the lane's column of a row that another lane has put
  __device__ __forceinline__ float get(int r) const {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];"
                 : "=f"(v)
                 : "r"(at + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4)
                 : "memory");
    return v;
  }
  // before the box is written again: its last copy has read it  (these two are for whole warps)
  __device__ __forceinline__ void open() const {
    if (lane == 0) tc::stores_read<0>();
    __syncwarp();
  }
  __device__ __forceinline__ void send(const CUtensorMap* map, int x, int y, int z, bool add) const {
    tc::fence_copies();
    __syncwarp();
    if (lane == 0) {
      if (add) tc::add_box(map, at, x, y, z);
      else tc::store_box(map, at, x, y, z);
      tc::close_stores();
    }
  }
};

struct Ring {
  uint32_t stages, empty;
  uint32_t full;       // of the pair's first block
  uint32_t full_here;
};

// A block's copies of a tile's operands.  (One thread issues them; what a step needs beside them counts, so that a kind
// has its own loop: with one loop for all, 1130 cycles a step of 520 on the tensor cores.)
template <XentKind KIND, int PAIRS>
__device__ __forceinline__ bool load_tile(const XentGemm& p, const XentWork& work, const XentTile& w, const Ring& r,
                                          int rank, unsigned& n, volatile int* gave_up) {
  const auto& g = p.g[work.shift][(p.turn + 1) & 1];
  const int an = w.m0 + rank * kBlockRows, bn = w.n0 + rank * (w.cols / 2);
  const uint32_t bytes = 2 * (kABytes + uint32_t(w.cols) * 64);
  const bool wide = w.cols > 128;
  const CUtensorMap* const ma = KIND == kLogits ? &p.hidden_rows : KIND == kHidden ? &g.rows : &g.cols;
  const CUtensorMap* const mb = KIND == kLogits ? &p.weight_rows : KIND == kHidden ? &p.weight_cols : &p.hidden_cols;
  const int b0 = KIND == kLogits ? work.next_v0 + bn : KIND == kHidden ? work.v0 : 0;
  for (int turn = 0; turn < PAIRS; ++turn) {
    // planes of the turns: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
    const int pa = PAIRS == 1 ? 0 : (0x001102 >> (4 * turn)) & 15;
    const int pb = PAIRS == 1 ? 0 : (0x010120 >> (4 * turn)) & 15;
    int k = w.k0 * kXentDepth;
    for (int i = 0; i < w.depth; ++i, ++n, k += kXentDepth) {
      const unsigned s = n % kStages;
      if (!tc::bar_wait(r.empty + 8 * s, (n / kStages + 1) & 1, gave_up)) return false;
      const uint32_t bar = r.full + 8 * s, a = r.stages + s * kStageBytes, b = a + kABytes;
      if (rank == 0) tc::bar_expect(r.full_here + 8 * s, bytes);
      else tc::bar_arrive_pair(bar);
      if (KIND == kWeight) {
        tc::load_box(ma, a, bar, an, k, pa);
        tc::load_box(ma, a + kBoxBytes, bar, an + 64, k, pa);
      } else {
        tc::load_box(ma, a, bar, k, an, pa);
      }
      if (KIND == kLogits) {
        tc::load_box(mb, b, bar, k, b0, pb);
      } else {
        tc::load_box(mb, b, bar, bn, b0 + k, pb);
        if (wide) tc::load_box(mb, b + kBoxBytes, bar, bn + 64, b0 + k, pb);
      }
    }
  }
  return true;
}

// The steps of a tile of the layer's gradient that bring the rests of the targets' entries, every kRestWarps-th of them from `which`
// on: of G's part of 64 tokens there is one value a token, which a warp writes to shared memory next to zeros.  (262144 tokens x
// 64 x 32 classes, gradients: 3.6 ms, 5.8 with one warp, 1.6 without the rests; 65536 x 768 x 5000: 3.00, 3.14 and 2.70.)
template <typename O>
__device__ __forceinline__ bool load_rests(const XentGemm& p, const XentWork& work, const XentTile& w, const Ring& r, int count,
                                           int rank, int which, int lane, unsigned n, volatile int* gave_up) {
  const int first = work.v0 + w.m0 + rank * kBlockRows, bn = w.n0 + rank * (w.cols / 2);
  int col[2];  // of this lane's two tokens, one step ahead
  float rest[2];
  const auto fetch = [&](int i) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int token = (w.rest0 + i) * kXentDepth + 32 * j + lane;
      const bool on = i < w.rests && token < count;
      col[j] = on ? p.target[token] - first : -1;
      rest[j] = on ? p.rest[token] : 0.f;
    }
  };
  fetch(which);
  for (int i = which; i < w.rests; i += kRestWarps) {
    const unsigned s = (n + i) % kStages;
    if (!__all_sync(kAll, tc::bar_wait(r.empty + 8 * s, ((n + i) / kStages + 1) & 1, gave_up))) return false;
    const uint32_t bar = r.full + 8 * s, a = r.stages + s * kStageBytes, b = a + kABytes;
#pragma unroll 8
    for (uint32_t at = lane * 16; at < kABytes; at += 512)
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(a + at), "r"(0) : "memory");
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = 32 * j + lane, c = col[j];
      if (c < 0 || c >= kBlockRows) continue;
      const O v = from_f32<O>(rest[j]);
      asm volatile("st.shared.u16 [%0], %1;" ::"r"(a + (c >> 6) * kBoxBytes + row * 128 +
                                                   ((((c & 63) >> 3) ^ (row & 7)) << 4) + (c & 7) * 2),
                   "h"(reinterpret_cast<const uint16_t&>(v))
                   : "memory");
    }
    fetch(i + kRestWarps);
    tc::fence_copies();
    __syncwarp();
    if (lane == 0) {
      const int token = (w.rest0 + i) * kXentDepth;
      if (rank == 0) tc::bar_expect(r.full_here + 8 * s, 2 * uint32_t(w.cols) * 64);
      else tc::bar_release_pair(bar);
      tc::load_box(&p.hidden_cols, b, bar, bn, token, 0);
      if (w.cols > 128) tc::load_box(&p.hidden_cols, b + kBoxBytes, bar, bn + 64, token, 0);
    }
  }
  return true;
}

template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kXentThreads, 1) k_xent(const __grid_constant__ XentGemm p) {
  using O = Operand<T>;
  constexpr int kPairs = std::is_same_v<T, float> ? 6 : 1;
  extern __shared__ unsigned char ring_[];
  __shared__ alignas(8) uint64_t bars[2 * kStages + 5];
  __shared__ uint32_t tmem_at;
  __shared__ int gave_up_;
  __shared__ unsigned loaded_;  // steps that the copying warp has come to, before each tile with rests
  volatile unsigned* loaded = &loaded_;
  volatile int* gave_up = &gave_up_;
  const uint32_t ring = (tc::smem_of(ring_) + 1023) & ~1023u;
  const uint32_t full = tc::smem_of(bars), empty = full + 8 * kStages, done = empty + 8 * kStages,
                 taken = done + 16, drained = taken + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = int(tc::pair_rank());
  if (threadIdx.x == 0) {
    gave_up_ = 0;
    loaded_ = 0;
    for (int i = 0; i < kStages; ++i) {
      tc::bar_init(full + 8 * i, 2);  // a thread of either block
      tc::bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::bar_init(done + 8 * i, 1);
      tc::bar_init(taken + 8 * i, 2 * kOutWarps);
    }
    tc::bar_init(drained, 1);
    tc::bar_init_fence();
  }
  if (warp == kOutWarps) tc::tmem_alloc(tc::smem_of(&tmem_at), 512);
  tc::fence_before();
  __syncthreads();
  tc::pair_sync();
  tc::fence_after();
  take_turn();
  const uint32_t tmem = tmem_at;
  const int count = *p.count, pairs = int(gridDim.x / 2), pair = int(blockIdx.x / 2);
  const XentWork work(p, count, pairs, BACKWARD, kPairs > 1);

  // Registers go where the sums are held: 128 x 72 + 256 x 216 of the launch's 384 x 168.
  const auto drain = [] {  // nothing may land in shared memory that the block has left: copies take microseconds
    const uint64_t start = tc::clock_ns();
    while (tc::clock_ns() - start < tc::kDrainNs) {
    }
  };
  if (warp >= kOutWarps) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == kOutWarps) {
    const Ring ring_of{ring, empty, tc::of_first(full), full};
    unsigned n = 0;  // steps so far
    bool ok = true;
    for (long long t = pair; t < work.all && ok; t += pairs) {
      const XentTile w = work.tile(p, t);
      if constexpr (BACKWARD && kPairs == 1)
        if (w.rests) {
          if (lane == 0) {
            __threadfence_block();
            *loaded = n;
          }
          ok = load_rests<O>(p, work, w, ring_of, count, rank, 0, lane, n, gave_up);
          n += unsigned(w.rests);
        }
      if (ok && lane == 0) {
        unsigned m = n;
        if (w.kind == kLogits) ok = load_tile<kLogits, kPairs>(p, work, w, ring_of, rank, m, gave_up);
        else if (w.kind == kHidden) ok = load_tile<kHidden, kPairs>(p, work, w, ring_of, rank, m, gave_up);
        else ok = load_tile<kWeight, kPairs>(p, work, w, ring_of, rank, m, gave_up);
      }
      n += unsigned(w.depth * kPairs);
      ok = __all_sync(kAll, ok);
    }
    if (!ok && lane == 0) drain();
    __syncwarp();
  } else if (warp == kOutWarps + 1) {
    if (lane == 0 && rank == 0) {
      unsigned n = 0, turn = 0;
      bool ok = true;
      for (long long t = pair; t < work.all && ok; t += pairs) {
        const XentTile w = work.tile(p, t);
        const bool a_mn = w.kind == kWeight, b_mn = w.kind != kLogits;
        const uint32_t ins = tc::instruction(std::is_same_v<O, __nv_bfloat16>, kXentRows, w.cols, a_mn, b_mn);
        const uint32_t a_step = a_mn ? 2048 : 32, b_step = b_mn ? 2048 : 32;
        const int steps = w.depth * kPairs + w.rests;
        int i = 0;
        do {  // an accumulator: the whole sum, or parts of it
          const unsigned buf = turn & 1;
          ok = tc::bar_wait(taken + 8 * buf, (turn / 2 + 1) & 1, gave_up);
          if (!ok) break;
          tc::fence_after();
          const int end = i + part_of<(kPairs > 1)>(w.kind, i, w.depth, steps);
          for (int j = 0; i < end; ++j, ++i, ++n) {
            const unsigned s = n % kStages;
            ok = tc::bar_wait(full + 8 * s, (n / kStages) & 1, gave_up);
            if (!ok) break;
            if (i < w.rests) tc::bar_acquire_pair(full + 8 * s, (n / kStages) & 1);  // (threads of both blocks wrote operands)
            tc::fence_after();
            const uint32_t a = ring + s * kStageBytes, b = a + kABytes;
#pragma unroll
            for (int k = 0; k < kXentDepth / 16; ++k)
              tc::mma(tmem + buf * kXentCols, tc::operand(a + k * a_step), tc::operand(b + k * b_step), ins,
                      j > 0 || k > 0);
            tc::commit(empty + 8 * s);
          }
          if (!ok) break;
          tc::commit(done + 8 * buf);
          ++turn;
        } while (i < steps);
      }
      if (!ok) {  // the products under way end before the tensor memory is given back
        tc::commit(drained);
        (void)tc::bar_wait(drained, 0, gave_up, tc::kDrainNs);
      }
    }
    __syncwarp();
  } else if constexpr (BACKWARD && kPairs == 1) {
    const Ring ring_of{ring, empty, tc::of_first(full), full};
    unsigned n = 0;
    bool ok = true;
    for (long long t = pair; t < work.weight && ok; t += pairs) {  // (no rests in the tiles behind)
      const XentTile w = work.tile(p, t);
      const int which = warp - kOutWarps - 1;
      if (which < w.rests) {
        // (a place's barrier tells of its last use only: the uses before these steps have to be under way)
        ok = __all_sync(kAll, tc::count_wait(loaded, n, gave_up)) &&
             load_rests<O>(p, work, w, ring_of, count, rank, which, lane, n, gave_up);
      }
      n += unsigned(w.rests + w.depth);
    }
    if (!ok && lane == 0) drain();
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int quarter = warp & 3, half = warp >> 2;
    const float back = BACKWARD ? p.scale[1] : 1.f;
    const uint32_t box = ring + kStages * kStageBytes + warp * kOutBytes;
    const CUtensorMap* const g_out = &p.g[work.shift][p.turn & 1].out;
    unsigned turn = 0;
    bool ok = true;
    for (long long t = pair; t < work.all && ok; t += pairs) {
      const XentTile w = work.tile(p, t);
      const int row0 = w.m0 + rank * kBlockRows + quarter * 32, row = row0 + lane;
      const int cols = w.cols / 2, n0 = w.n0 + half * cols;
      const int steps = w.depth * kPairs + w.rests;
      int target = -1;
      RowLse lse;
      float coef = 0.f, times = 0.f;
      if (w.kind == kLogits) {
        target = p.target[row];
        if constexpr (BACKWARD) {
          lse.set(p.lse[row]);
          coef = p.coef[row];
          times = coef * lse.scale;
        }
      }
      RowStats stats;
      // 32 columns of the finished result
      const auto put = [&](int c, float(&v)[32]) {
        const int col = n0 + c;
        if constexpr (!BACKWARD) {
          stats.add(p, row, target, col, v);
        } else if (w.kind == kLogits) {
          if (col >= work.piece) return;  // (all lanes, here and below: no box begins outside of what it is stored to)
          const int hit = target - (work.next_v0 + col);
          const int valid = row < count ? work.next_cols - col : 0;
          const bool mine = hit >= 0 && hit < 32;
          float x = 0.f;
          if (mine) {
#pragma unroll
            for (int i = 0; i < 32; ++i) x = i == hit ? v[i] : x;
            x = (exp_pair(x, x, lse.base).x * lse.scale - 1.f) * coef;
            if constexpr (kPairs == 1) p.rest[row] = x - rounded<O>(x);
          }
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 e = mul2(exp_pair(v[i], v[i + 1], lse.base), both(times));
            v[i] = e.x;
            v[i + 1] = e.y;
          }
          if (mine) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = i == hit ? x : v[i];
          }
          if (valid < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = i < valid ? v[i] : 0.f;
          }
          if constexpr (kPairs == 1) {
            const OutBox<O> out{box, lane};
            const bool second = c & 32;  // half of a box of 64 columns
            if (!second) out.open();
            out.put(second ? 4 : 0, v);
            if (second) out.send(g_out, col - 32, row0, 0, false);
          } else {
#pragma unroll
            for (int plane = 0; plane < 3; ++plane) {
              const OutBox<O, 64> out{box, lane};
              out.open();
              out.put(0, v);
              out.send(g_out, col, row0, plane, false);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] -= rounded<O>(v[i]);
            }
          }
        } else if (w.kind == kHidden) {
          if (col >= p.d) return;
          if (!steps) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          const OutBox<float> out{box, lane};
          out.open();
          out.put(0, v);
          out.send(&p.sum_out, col, w.part * work.row_tiles * kXentRows + row0, 0, p.turn > 1);
        } else {
          if ((col & ~63) >= p.d || row0 >= work.rows) return;
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = steps ? v[i] * back : 0.f;
          if (p.box_dweight) {
            constexpr int kWide = 128 / int(sizeof(T));  // columns of a box
            const OutBox<T> out{box, lane};
            const bool second = c & (kWide - 32);
            if (!second) out.open();
            out.put(second ? 4 : 0, v);
            if (second || (kWide == 32 && col < p.d)) out.send(&p.dweight_out, col & ~(kWide - 1), work.v0 + row0, 0, false);
          } else {  // rows that begin anywhere: turned in shared memory, so that a warp's accesses lie together
            const OutBox<float> turned{box, lane};
            turned.open();
            turned.put(0, v);
            __syncwarp();
            T* to = static_cast<T*>(p.dweight) + (long long)(work.v0 + row0) * p.d + col + lane;
            const int valid = col + lane < p.d ? min(32, work.rows - row0) : 0;
#pragma unroll 8
            for (int r = 0; r < valid; ++r, to += p.d) *to = from_f32<T>(turned.get(r));
            __syncwarp();
          }
        }
      };
      const auto await = [&] {
        ok = __all_sync(kAll, tc::bar_wait(done + 8 * (turn & 1), (turn / 2) & 1, gave_up));
        tc::fence_after();
        return ok;
      };
      const auto give = [&] {
        tc::fence_before();
        __syncwarp();
        if (lane == 0) tc::bar_arrive_pair(tc::of_first(taken + 8 * (turn & 1)));
        ++turn;
      };
      const auto at = [&](int c) {
        return tmem + (turn & 1) * kXentCols + half * cols + c + (uint32_t(quarter * 32) << 16);
      };
      float acc[kXentCols / 64][32];
      if (!await()) break;
#pragma unroll
      for (int j = 0; j < kXentCols / 64; ++j)
        if (32 * j < cols) tc::tmem_load32(at(32 * j), acc[j]);
#pragma unroll
      for (int j = 0; j < kXentCols / 64; ++j) tc::tmem_wait(acc[j]);
      give();
      for (int i = part_of<(kPairs > 1)>(w.kind, 0, w.depth, steps); i < steps;
           i += part_of<(kPairs > 1)>(w.kind, i, w.depth, steps)) {
        if (!await()) break;
        float v[2][32];
        tc::tmem_load32(at(0), v[0]);
#pragma unroll
        for (int j = 0; j < kXentCols / 64; ++j) {
          if (32 * j >= cols) break;
          tc::tmem_wait(v[j & 1]);
          if (j + 1 < kXentCols / 64 && 32 * (j + 1) < cols) tc::tmem_load32(at(32 * (j + 1)), v[(j + 1) & 1]);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 s = add2(make_float2(acc[j][e], acc[j][e + 1]), make_float2(v[j & 1][e], v[j & 1][e + 1]));
            acc[j][e] = s.x;
            acc[j][e + 1] = s.y;
          }
        }
        give();
      }
      if (!ok) break;
#pragma unroll
      for (int j = 0; j < kXentCols / 64; ++j)
        if (32 * j < cols) put(32 * j, acc[j]);
      if constexpr (!BACKWARD)
        p.part[(long long)row * p.parts + w.part * 2 + half] = make_float2(stats.top, stats.total);
      __syncwarp();
    }
    if (lane == 0) tc::stores_done();
    __syncwarp();
  }
  tc::fence_before();
  __syncthreads();
  tc::pair_sync();  // the other block's products read this one's shared memory
  if (warp == kOutWarps) tc::tmem_free(tmem, 512);
  if (threadIdx.x == 0 && gave_up_) atomicExch(p.status, EFCP_ETIMEOUT);
}

// What comes before the products: which tokens have a target, in order; their rows of H, one behind the other (and
// zeros up to whole tiles), as the copies of tiles want them; backward also the factors on their gradients, times a
// power of two that brings the largest near 1 (near 2^14 for fp16, whose probabilities would vanish otherwise); and
// zeros for what belongs to the other tokens.  Where the rests of the targets' entries are asked for (p.bounds) the order goes by
// the targets' tiles first, so that a tile of rows of W meets its targets in few steps (2458 tokens x 30522 classes: in one or two of
// 39; in the tokens' own order it would be 16).
//
// A block takes a run of tokens.  It counts those with a target before its own by itself, so that one launch is
// enough: all targets pass through every block, 8 bytes for each row of H.
template <typename T>
__global__ void __launch_bounds__(512) k_xent_prepare(const XentPrep p, bool backward, int per) {
  take_turn();
  using O = Operand<T>;
  constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 1;
  constexpr bool kHalf = std::is_same_v<T, __half>;
  __shared__ int before_, all_, places[512 / 32], tokens[512], rows[512];
  __shared__ int bucket[512], bucket_all[kXentBuckets], bucket_at[kXentBuckets];  // (sorted)
  __shared__ unsigned most_;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long lo = (long long)blockIdx.x * per, hi = min(p.tokens, lo + per);
  if (threadIdx.x == 0) {
    before_ = all_ = 0;
    most_ = 0;
  }
  __syncthreads();
  int before = 0, all = 0;
  float big = 0.f;
  const bool each = backward && p.reduction == 0, sorted = p.bounds;
  const auto bucket_of = [&](long long t) { return t >= 0 && t < p.vocab ? int(t / kXentRows) >> p.wide : 0; };
  if (sorted) {
    for (int i = threadIdx.x; i < kXentBuckets; i += 512) bucket_all[i] = bucket_at[i] = 0;
    __syncthreads();
  }
  constexpr int kAhead = 8;  // loads on their way: counting in shared memory would wait for each
  for (long long i0 = threadIdx.x; i0 < p.tokens; i0 += 512 * kAhead) {
    long long t[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) t[k] = i0 + 512 * k < p.tokens ? p.targets[i0 + 512 * k] : p.ignore;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long long i = i0 + 512 * k;
      const bool used = t[k] != p.ignore;
      all += used;
      before += used && i < lo;
      if (each && used) {
        const float g = fabsf(p.grad[i * p.grad_step]);
        if (g < INFINITY) big = fmaxf(big, g);
      }
    }
    if (sorted) {  // (whole numbers: any order)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (t[k] == p.ignore) continue;
        atomicAdd(&bucket_all[bucket_of(t[k])], 1);
        if (i0 + 512 * k < lo) atomicAdd(&bucket_at[bucket_of(t[k])], 1);
      }
    }
  }
  before = __reduce_add_sync(kAll, before);
  all = __reduce_add_sync(kAll, all);
  big = lanes_max(big, 32);
  if (lane == 0) {
    atomicAdd(&before_, before);  // (whole numbers: any order)
    atomicAdd(&all_, all);
    atomicMax(&most_, __float_as_uint(big));  // (of values that are not negative the bits are in order)
  }
  __syncthreads();
  if (sorted) {  // where the block's next token of each bucket goes
    const int k = 2 * threadIdx.x, two = bucket_all[k] + bucket_all[k + 1];
    int sum = two;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int other = __shfl_up_sync(kAll, sum, o);
      if (lane >= o) sum += other;
    }
    if (lane == 31) places[warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += places[w];
    if (blockIdx.x == 0) {
      p.bounds[k] = sum - two;
      p.bounds[k + 1] = sum - two + bucket_all[k];
      if (k + 2 == kXentBuckets) p.bounds[k + 2] = sum;
    }
    bucket_at[k] += sum - two;
    bucket_at[k + 1] += sum - two + bucket_all[k];
    __syncthreads();
  }
  all = all_;
  int at = before_;
  const int padded = (all + kXentRows - 1) / kXentRows * kXentRows;
  float one = 0.f, up = 1.f;
  if (backward) {
    if (!each) {
      one = p.grad[0] * (p.reduction == 1 ? 1.f / float(all) : 1.f);
      big = fabsf(one) < INFINITY ? fabsf(one) : 0.f;
    } else {
      big = __uint_as_float(most_);
    }
    const int e = big > 0.f ? max(-100, min(100, ilogbf(big))) : 0, shift = kHalf ? 14 : 0;
    up = scalbnf(1.f, shift - e);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      p.scale[0] = up;
      p.scale[1] = scalbnf(1.f, e - shift);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.count = all;
  const int chunks = (p.d + 255) / 256;
  const auto copy = [&](long long token, int place, int c0) {  // 256 columns of a row  (a warp)
    const T* from = static_cast<const T*>(p.hidden) + token * p.hidden_row;
    O* to = static_cast<O*>(p.hidden_packed) + place * p.packed_row;
    if (kPlanes == 1 && reinterpret_cast<uintptr_t>(from) % 16 == 0 && p.d % 8 == 0) {
      const int c = c0 + lane * 8;
      if (c < p.d) *reinterpret_cast<uint4*>(to + c) = *reinterpret_cast<const uint4*>(from + c);
    } else {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = c0 + 32 * j + lane < p.d ? to_f32(from[c0 + 32 * j + lane]) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = c0 + 32 * j + lane;
        if (c >= p.d) continue;
        O v[kPlanes];
        split<O, kPlanes>(x[j], v);
#pragma unroll
        for (int k = 0; k < kPlanes; ++k) to[k * p.hidden_plane + c] = v[k];
      }
    }
  };
  for (long long base = lo; base < hi; base += 512) {
    const long long i = base + threadIdx.x;
    const long long t = i < hi ? p.targets[i] : p.ignore;
    const bool used = t != p.ignore;
    const unsigned mask = __ballot_sync(kAll, used);
    if (lane == 0) places[warp] = __popc(mask);
    if (sorted) bucket[threadIdx.x] = used ? bucket_of(t) : -1;
    __syncthreads();
    int first = 0, here = 0;  // tokens with a target before this warp's; of the block
    for (int k = 0; k < 512 / 32; ++k) {
      if (k < warp) first += places[k];
      here += places[k];
    }
    const int local = first + __popc(mask & ((1u << lane) - 1));
    int place = at + local;
    if (sorted && used) {
      place = bucket_at[bucket[threadIdx.x]];
      for (int k = 0; k < threadIdx.x; ++k) place += bucket[k] == bucket[threadIdx.x];
    }
    if (used) {
      tokens[local] = int(i);
      rows[local] = place;
    }
    if (i < hi) {
      if (p.place) p.place[i] = used ? place : -1;
      if (used) {
        const bool in = t >= 0 && t < p.vocab;
        p.order[place] = int(i);
        p.target[place] = in ? int(t) : -1;
        if (backward) {
          const float g = each ? p.grad[i * p.grad_step] : one;
          if (p.rest) p.rest[place] = 0.f;
          p.coef[place] = in ? g * up : __int_as_float(0x7FC00000);
          p.lse[place] = p.lse_in[i];
        }
      } else {
        if (p.losses && !p.reduction) p.losses[i] = 0.f;
        if (p.lse_out) p.lse_out[i] = 0.f;
      }
    }
    __syncthreads();
    if (sorted && used) atomicAdd(&bucket_at[bucket[threadIdx.x]], 1);
#pragma unroll 2
    for (int k = warp; k < here * chunks; k += 512 / 32) {
      const int token = k / chunks;
      copy(tokens[token], rows[token], (k - token * chunks) * 256);
    }
    at += here;
    __syncthreads();
  }
  if (blockIdx.x == gridDim.x - 1) {
    for (int i = all + threadIdx.x; i < padded; i += 512) {
      p.target[i] = -1;
      if (backward) p.coef[i] = p.lse[i] = 0.f;
    }
  }
  for (int i = all + int(blockIdx.x) * 16 + warp; i < padded; i += int(gridDim.x) * 16)
    for (int k = 0; k < kPlanes; ++k) {
      O* to = static_cast<O*>(p.hidden_packed) + k * p.hidden_plane + (long long)i * p.packed_row;
      for (int c = lane * 8; c < p.packed_row; c += 256) *reinterpret_cast<uint4*>(to + c) = make_uint4(0, 0, 0, 0);
    }
}

// W as the copies of tiles want it, where it does not lie so.  A warp takes 256 columns of a row, a lane pairs of them.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_pack(const XentPrep p) {
  take_turn();
  using O = Operand<T>;
  constexpr int kPlanes = std::is_same_v<T, float> ? 3 : 1;
  const int lane = threadIdx.x & 31, chunks = (p.d + 255) / 256;
  const long long warps = (long long)gridDim.x * 8, all = (long long)p.vocab * chunks;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < all; i += warps) {
    const long long row = i / chunks;
    const int c0 = int(i - row * chunks) * 256 + 2 * lane;
    const T* from = static_cast<const T*>(p.weight) + row * p.weight_row;
    O* to = static_cast<O*>(p.weight_packed) + row * p.packed_row;
    float v[4][2];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j) v[k][j] = c0 + 64 * k + j < p.d ? to_f32(from[c0 + 64 * k + j]) : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = c0 + 64 * k;
      if (c >= p.d) continue;  // (rows are a multiple of eight long: the second of a pair has its place)
      O a[kPlanes], b[kPlanes];
      split<O, kPlanes>(v[k][0], a);
      split<O, kPlanes>(v[k][1], b);
#pragma unroll
      for (int j = 0; j < kPlanes; ++j) {
        Pack<O, 2> two;
        two.v[0] = a[j];
        two.v[1] = b[j];
        *reinterpret_cast<Pack<O, 2>*>(to + j * p.weight_plane + c) = two;
      }
    }
  }
}

// The gradient of H from its parts; zeros for tokens without a target.  A warp takes 128 columns of a row.  The target's entry of
// G is by far a row's largest, and what its rounding to 16 bits left is added here.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_finish(const XentPrep p) {
  take_turn();
  const int lane = threadIdx.x & 31, chunks = (p.d + 127) / 128;
  const int row_tiles = (*p.count + kXentRows - 1) / kXentRows;
  const int splits =
      xent_splits(row_tiles, p.d_tiles, p.piece << xent_shift(row_tiles, p.tiles, p.shifts), p.pairs, std::is_same_v<T, float>);
  const long long part = (long long)row_tiles * kXentRows * p.sum_row, all = p.tokens * chunks;
  const float back = p.scale[1];
  const bool vec = reinterpret_cast<uintptr_t>(p.dhidden) % 16 == 0 && p.d % 4 == 0;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < all; i += (long long)gridDim.x * 8) {
    const long long token = i / chunks;
    const int c = int(i - token * chunks) * 128 + lane * 4;
    if (c >= p.d) continue;
    const int place = p.place[token];
    T* to = static_cast<T*>(p.dhidden) + token * p.d;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (place >= 0) {
      const float* from = p.sum + place * p.sum_row + c;  // (rows are a multiple of 32 long)
      for (int k0 = 0; k0 < splits; k0 += 8) {
        float4 o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          o[k] = k0 + k < splits ? *reinterpret_cast<const float4*>(from + (k0 + k) * part) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v.x += o[k].x; v.y += o[k].y; v.z += o[k].z; v.w += o[k].w;
        }
      }
      const float rest = p.rest ? p.rest[place] : 0.f;
      if (rest != 0.f) {
        const T* w = static_cast<const T*>(p.layer) + p.target[place] * p.weight_row + c;
        v.x += rest * to_f32(w[0]);
        if (c + 1 < p.d) v.y += rest * to_f32(w[1]);
        if (c + 2 < p.d) v.z += rest * to_f32(w[2]);
        if (c + 3 < p.d) v.w += rest * to_f32(w[3]);
      }
    }
    Pack<T, 4> a;
    a.v[0] = from_f32<T>(v.x * back); a.v[1] = from_f32<T>(v.y * back);
    a.v[2] = from_f32<T>(v.z * back); a.v[3] = from_f32<T>(v.w * back);
    if (vec) {
      *reinterpret_cast<Pack<T, 4>*>(to + c) = a;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < p.d) to[c + j] = a.v[j];
    }
  }
}

template <typename T, bool BACKWARD>
cudaError_t xent_launch(const XentGemm& p, unsigned pairs, cudaStream_t st) {
  const auto kern = k_xent<T, BACKWARD>;
  // (the same value every time: a kernel's limit belongs to the device, not to this launch)
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kXentSmem));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs);
  cfg.blockDim = dim3(kXentThreads);
  cfg.dynamicSmemBytes = kXentSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <typename T>
cudaError_t xent_prepare(const XentPrep& p, bool backward, int sms, cudaStream_t st) {
  // runs of tokens for two blocks on each SM
  const long long per = std::max<long long>(4, (p.tokens + 2 * sms - 1) / (2 * sms));
  const unsigned blocks = unsigned(std::max<long long>(1, (p.tokens + per - 1) / per));
  cudaError_t e = launch(k_xent_prepare<T>, Shape{blocks, 512, 0, 0}, st, p, backward, int(per));
  if (e != cudaSuccess || !p.weight) return e;
  const long long warps = (long long)p.vocab * ((p.d + 255) / 256);
  return launch(k_xent_pack<T>, Shape{unsigned(std::min<long long>(warps / 8 + 1, 8ll * sms)), 256, 0, 0}, st, p);
}

template <typename T>
cudaError_t xent_finish(const XentPrep& p, int sms, cudaStream_t st) {
  const long long warps = p.tokens * ((p.d + 127) / 128);
  return launch(k_xent_finish<T>, Shape{unsigned(std::min<long long>(warps / 8 + 1, 8ll * sms)), 256, 0, 0}, st, p);
}

}  // namespace
}  // namespace efcp
