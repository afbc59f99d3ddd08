// Attention under the mask of parallel groups: what its kernels share.
//
// A sequence has `ctx` context rows (keys only) and `groups` groups of R rows, a real one and R - 1 [MASK] rows.  A
// query row (index rho = t R + j within the sequence) sees
//   the context                       keys 0 .. ctx-1
//   the real rows of groups 0 .. t    keys x with x <= t
//   its own group's masks 1 .. j      group rows t R + 1 .. rho
// so its keys come in three kinds of tiles, and in each tile what a row sees is one range of columns.
#pragma once
#include "train_ops.cuh"

namespace ps {
namespace train {

enum TileKind { CTX = 0, REAL = 1, LOCAL = 2 };

// By value to the kernels.  Row offsets are those of the first group row (q0) and the first context row (kv0).
struct Seqs {
  int B, R;
  int ctx[PS_MAX_BATCH], groups[PS_MAX_BATCH];
  int q0[PS_MAX_BATCH + 1], kv0[PS_MAX_BATCH + 1];
  int tile0[PS_MAX_BATCH + 1];    // tiles (of the launch's kind) before the sequence
};

struct AttnArgs {
  int n_heads, n_kv, per;    // per: query heads of a key head
  int rows;                  // group rows
  float scale;
  const void *q, *k, *v;
  size_t ldq, ldk, ldv;
  void* out;
  size_t ldo;
  float* lse;
  const void* dout;
  size_t lddo;
  void *dq, *dk, *dv;
  size_t lddq, lddk, lddv;
  float* delta;              // [n_heads][rows] dout . out
  int* status;
};

__device__ __forceinline__ int seq_of_tile(const Seqs& s, int t) {
  int lo = 0, hi = s.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.tile0[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__host__ __device__ constexpr int div_up(int a, int b) { return (a + b - 1) / b; }
// Groups whose rows lie in one query tile of at most `rows` rows.
__host__ __device__ constexpr int groups_per_tile(int rows, int R) { return rows / R; }

}  // namespace train
}  // namespace ps
