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
  int* any;                  // bf16, backward: whether a sum is not finite
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

// Keys up to which a bf16 row's delta = dout . out is formed from the probabilities instead, as sum_c p_c (dout . v_c).  out is
// rounded, and what that takes from delta a row with few keys has no small share of in its gradients: p (dP - delta) is the
// difference of near numbers where one of two keys has most of the weight (two rows of two keys: dq 1.0e-2 off
// relatively; 1.7e-3 with this).  With more keys the rounding of dS is by far the larger part.
constexpr int kExactKeys = 32;
__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
// delta of row rho of sequence b and head h from its n keys, by one warp.
template <class T, int D>
__device__ __noinline__ float delta_of_keys(const Seqs& s, const AttnArgs& a, int b, int rho, int h, int n) {
  const int lane = threadIdx.x & 31, R = s.R, t = rho / R, ctx = s.ctx[b];
  const size_t qr = (size_t)s.q0[b] + rho, kv0 = s.kv0[b], g0 = kv0 + ctx;
  const T *k = (const T*)a.k + (size_t)(h / a.per) * D, *v = (const T*)a.v + (size_t)(h / a.per) * D;
  const T *q_in = (const T*)a.q + qr * a.ldq + (size_t)h * D, *g_in = (const T*)a.dout + qr * a.lddo + (size_t)h * D;
  float q[D / 32], g[D / 32], sum = 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) {
    q[e] = wide(q_in[lane + 32 * e]);
    g[e] = wide(g_in[lane + 32 * e]);
  }
  const float lse = a.lse[(size_t)h * a.rows + qr];
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    const size_t row = c < ctx ? kv0 + c : (c <= ctx + t ? g0 + (size_t)(c - ctx) * R : g0 + (size_t)t * R + (c - ctx - t));
    float sc = 0.f, dp = 0.f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      sc = fmaf(q[e], wide(k[row * a.ldk + lane + 32 * e]), sc);
      dp = fmaf(g[e], wide(v[row * a.ldv + lane + 32 * e]), dp);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sc += __shfl_xor_sync(0xffffffffu, sc, o);
      dp += __shfl_xor_sync(0xffffffffu, dp, o);
    }
    sum = fmaf(exp2f((sc * a.scale - lse) * 1.4426950408889634f), dp, sum);
  }
  return sum;
}

__host__ __device__ constexpr int div_up(int a, int b) { return (a + b - 1) / b; }
// Groups whose rows lie in one query tile of at most `rows` rows.
__host__ __device__ constexpr int groups_per_tile(int rows, int R) { return rows / R; }

}  // namespace train
}  // namespace ps
