// What the two ways of the LM-head loss share: buffers of a call and the kernels around the matrix products.
#pragma once
#include "train_ops.cuh"

namespace ps {
namespace train {

// Rows that count are numbered 0 .. n-1 in order ("compact" rows): a row whose label lies outside the vocabulary takes
// no part in any product, so that whatever its x holds reaches nothing.
struct LossBuf {
  int* n;                // [1] rows that count
  int* row_of;           // [rows] row of a compact row
  int* slot;             // [rows] compact row of a row, -1: it counts for nothing
  int* label;            // [rows_pad] of compact rows
  float *lse, *up;       // [rows_pad] of compact rows: lse and dloss (backward)
  void* x;               // [rows_pad][hidden] compact rows, dtype
  // forward: per vocabulary tile and compact row the maximum and the sum of exponentials against it, the label's logit left out
  float2* part;          // [rows_pad][tiles]
  float* own;            // [rows_pad] logit of the label as the product formed it
  float* picked;         // [rows_pad] logit of the label in single precision
  // backward
  void* g;               // [rows_pad][piece] gradient of a piece's logits
  float* acc;            // [splits][rows_pad][hidden] dx so far
  size_t bytes;
};

struct LossPlan {
  bool tc;               // bf16: the tensor-core kernels (lm_loss_tc.cu)
  int rows, rows_pad, hidden, vocab;
  int tile_v, tiles;     // vocabulary rows of a tile of the forward pass
  int piece;             // vocabulary rows of a piece of the backward pass
  int splits;            // parts of a piece that dx is summed over (tensor cores: at most, see dx_splits)
};

struct LossArgs {
  LossPlan p;
  LossBuf b;
  const void* w;
  void* dw;
  bool want_dx;
  int* status;
};

// Parts of a piece's kb k blocks that the tensor cores' dx is dealt in: what a pair then works in sequence is least, in k blocks and
// kTileCost of them for each tile's beginning and end.  (180 tiles on 74 pairs are three waves, of which two parts each make
// five half ones: 13B, 2253 rows that count, the whole of loss and dx 1.91 -> 1.88 ms.)
constexpr int kMaxSplits = 4, kTileCost = 6, kLossTile = 256;
__host__ __device__ inline int dx_splits(int rows, int hidden, int kb, int pairs) {
  const int tiles = ((rows + kLossTile - 1) / kLossTile) * ((hidden + kLossTile - 1) / kLossTile);
  int best = 1, least = 0;
  for (int s = 1; s <= kMaxSplits; ++s) {
    const int cost = (tiles * s + pairs - 1) / pairs * ((kb + s - 1) / s + kTileCost);
    if (s == 1 || cost < least) { best = s; least = cost; }
  }
  return best;
}

// ---- lm_loss_tc.cu
cudaError_t loss_forward_tc(const LossArgs& a, cudaStream_t st);
cudaError_t loss_piece_tc(const LossArgs& a, int v0, int nv, cudaStream_t st);

}  // namespace train
}  // namespace ps
