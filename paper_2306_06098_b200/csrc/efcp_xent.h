// Between the host side of the linear cross-entropy calls (efcp_cross_entropy.cu) and their kernels
// (efcp_xent.cuh), which are compiled once per element type.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace efcp {

// Products of tiles: what is multiplied, and what becomes of the sums.
enum XentMode {
  kXentStats,    // logits = H W^T: largest value and sum of exponentials of a row's part, the target's logit
  kXentGrad,     // logits once more: gradient of the logits of a piece of the vocabulary
  kXentHidden,   // gradient of H, added up over the pieces
  kXentWeight,   // gradient of the piece's rows of W
};

constexpr int kXentRows = 128, kXentCols = 256, kXentDepth = 64;  // a tile, and a step along the sum

struct XentGemm {
  CUtensorMap a, b;
  const int* count;    // tokens that have a target
  const int* order;    // their places in the batch
  const int* target;   // their targets, -1: out of range
  const float* lse;    // logarithm of the sum of exponentials (by the tokens' order here)
  const float* coef;   // factor on a token's gradient
  const float* scale;  // [0]: the factor that coef holds, [1]: its inverse
  float2* part;        // statistics, a row of `parts` for each token
  float* target_logit;
  void* g;                        // gradient of the logits: planes of rows of the piece's columns
  long long g_row, g_plane;       // in elements
  float* sum;                     // of the pieces before, fp32, sum_row elements a row
  long long sum_row;
  void* out;                      // gradient of H or W
  long long out_row;
  int* status;
  int vocab, d;
  int v0, piece;     // columns v0 .. v0 + piece of the vocabulary (padded with zeros to g's width)
  int parts;
  int row_tiles;     // -1: of the tokens that have a target
  int col_tiles, col_tile;
  int depth;         // length of the sum, -1: the tokens
  int planes;        // 1, or 3 for fp32 values held as three bfloat16 ones
  int first, last;   // piece
  int vec_out;       // rows of out start on 16 bytes
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
  void* dhidden;       // rows without a target become zeros
};

cudaError_t xent_gemm_f32(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st);
cudaError_t xent_gemm_bf16(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st);
cudaError_t xent_gemm_f16(XentMode mode, const XentGemm& p, unsigned blocks, cudaStream_t st);
cudaError_t xent_prepare_f32(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_prepare_bf16(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_prepare_f16(const XentPrep& p, bool backward, int sms, cudaStream_t st);
cudaError_t xent_join(const XentPrep& p, int sms, cudaStream_t st);

}  // namespace efcp
