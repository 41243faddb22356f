// Between the host side of the linear cross-entropy calls (efcp_cross_entropy.cu) and their kernels
// (efcp_xent.cuh), which are compiled once per element type.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace efcp {

// A tile of a product (256 x up to 256, of a pair of blocks), and a step along the sum.
constexpr int kXentRows = 256, kXentCols = 256, kXentDepth = 64;
constexpr int kXentShifts = 3;
constexpr int kXentBuckets = 1024;  // of targets, at most
constexpr float kLog2e = 1.4426950408889634f;  // e^x = 2^(x log2(e)), up to this one's rounding: see k_xent_join
constexpr int kXentSplits = 32;  // parts of the sum over a piece that are added up apart, at most

// The products of tiles that a launch works on, in this order:
//   hidden   gradient of H from a piece's gradient of the logits, in parts, added to those of the pieces before
//   weight   gradient of the piece's rows of W
//   logits   forward: largest value and sum of exponentials of a row's part, and the target's logit;
//            backward: the gradient of the logits of the next piece
struct XentGemm {
  // operands whose inner dimension is that of the sum (rows of 64 in boxes of a block's share of a tile), and the
  // others (boxes of 64 x 64)
  CUtensorMap hidden_rows, weight_rows, hidden_cols, weight_cols;
  // results, stored in boxes of 32 rows of 128 bytes
  CUtensorMap sum_out, dweight_out;
  struct {
    CUtensorMap rows, cols, out;
  } g[kXentShifts + 1][2];  // the gradient of the logits, by the width of a piece
  const int* count;    // tokens that have a target
  const int* target;   // their targets, -1: out of range
  const float* lse;    // logarithm of the sum of exponentials (by the tokens' order here)
  const float* coef;   // factor on a token's gradient
  const float* scale;  // [0]: the factor that coef holds, [1]: its inverse
  float* rest;         // what the rounding of G left of the targets' entries (16 bits)
  const int* bounds;   // tokens lie in the order of their targets' tiles of rows of W: where the tokens of a bucket of
  int wide;            // 2^wide tiles begin (16 bits)
  float2* part;        // statistics, a row of `parts` for each token
  float* target_logit;
  void* dweight;
  int* status;
  int vocab, d;
  int parts;
  int d_tiles, d_tile;
  int hidden, weight;                  // which of the products of a piece are wanted
  int turn;                            // the launch works on piece turn - 1 and the logits of piece turn
  int col_tiles, col_tile;             // of logits (forward; of a piece not widened)
  int piece, tiles, shifts;            // see xent_shift
  int box_dweight;                     // rows of dweight start on 16 bytes: it can be stored in boxes
};

struct XentPrep {
  const long long* targets;
  long long tokens, ignore;
  int vocab, d;
  const void* hidden;
  long long hidden_row;
  const void* weight;  // to be packed, or null
  long long weight_row;
  void *hidden_packed, *weight_packed;  // planes of rows of `packed_row` elements
  long long packed_row, hidden_plane, weight_plane;
  int *count, *order, *target;
  float *lse, *coef, *scale, *target_logit;
  const float2* part;
  int parts;
  int reduction;       // 0 none, 1 mean, 2 sum
  const float* grad;   // of the losses, or of the one value
  long long grad_step;
  const float* lse_in;
  float *losses, *lse_out, *each;  // each: losses by order, to be added up
  float* rest;                     // see XentGemm
  const void* layer;               // the weight as it was given
  int* place;                      // a token's place in the order, -1: none
  int* bounds;                     // see XentGemm, kXentBuckets + 1 of them; null: not wanted
  int wide;
  const float* sum;                // gradient of H: parts of the whole tiles' rows, sum_row elements each
  long long sum_row;
  int d_tiles, piece, tiles, shifts, pairs;
  void* dhidden;
};

// The calls for up to eight tokens (efcp_xent_few.cuh).
constexpr int kFewTokens = 8;
struct XentFew {
  const long long* targets;
  long long ignore;
  int tokens, vocab, d;
  int padded;  // d up to a multiple of 256
  int blocks;
  int reduction;
  const void* hidden;
  long long hidden_row;
  const void* weight;
  long long weight_row;
  // forward
  float2* part;  // a token's statistics, one a block
  float* target_logit;
  float *losses, *lse_out;
  // backward
  const float* grad;
  long long grad_step;
  const float* lse_in;
  float* g;     // the logits' gradient, 4 or 8 tokens of a row of the weight side by side
  float* sums;  // of the gradient of H: for each token `ranges` rows of `padded`  (null: not wanted)
  int ranges;   // blocks that share a set of columns
  void *dhidden, *dweight;
};

// How often a piece's columns are doubled.  The buffers hold `piece` columns for all tokens, `tiles` tiles of rows; how many
// of them have a target is known on the device alone, and with fewer rows a piece is wider: fewer launches do something.
__host__ __device__ inline int xent_shift(int row_tiles, int tiles, int shifts) {
  int s = 0;
  while (s < shifts && row_tiles <= (tiles >> (s + 1))) ++s;
  return s;
}

// How many parts the sum over a piece is cut into for the gradient of H: as many as give every pair of blocks two
// tiles, up to eight, none shorter than 16 steps.  With a few tiles of H only (up to four on a B200), as many as give every
// pair one, and shorter ones where a step is six products.  (17 tokens x 64 x 933 fp32, gradients: 39 us, 60 with eight at
// most; but 1003 x 509 x 10007 with more than eight 275 us, and 239.)
__host__ __device__ inline int xent_splits(int row_tiles, int d_tiles, int piece, int pairs, bool six) {
  const int tiles = row_tiles * d_tiles;
  if (tiles == 0) return 1;
  const bool lone = 16 * tiles <= pairs;
  const int least = kXentDepth * (lone && six ? 4 : 16), deepest = (piece + least - 1) / least;
  int s = ((lone ? 1 : 2) * pairs + tiles - 1) / tiles;
  s = s < deepest ? s : deepest;
  const int most = lone ? kXentSplits : 8;
  return s < 1 ? 1 : s < most ? s : most;
}

cudaError_t xent_gemm_f32(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st);
cudaError_t xent_gemm_bf16(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st);
cudaError_t xent_gemm_f16(bool backward, const XentGemm& p, unsigned pairs, cudaStream_t st);
cudaError_t xent_prepare_f32(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_prepare_bf16(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_prepare_f16(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_finish_f32(const XentPrep& p, int sms, cudaStream_t st);
cudaError_t xent_finish_bf16(const XentPrep& p, int sms, cudaStream_t st);
cudaError_t xent_finish_f16(const XentPrep& p, int sms, cudaStream_t st);
cudaError_t few_launch_f32(const XentFew& p, bool vec, bool backward, cudaStream_t st);
cudaError_t few_launch_bf16(const XentFew& p, bool vec, bool backward, cudaStream_t st);
cudaError_t few_launch_f16(const XentFew& p, bool vec, bool backward, cudaStream_t st);
cudaError_t xent_join(const XentPrep& p, int sms, cudaStream_t st);

}  // namespace efcp
