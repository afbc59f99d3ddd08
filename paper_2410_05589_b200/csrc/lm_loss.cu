// Softmax cross entropy of the LM head (ps_lm_loss, ps_lm_loss_backward) over pieces of the vocabulary.
//
//   s = x W^T,  lse = log sum_v exp s_v,  loss = lse - s_label
//   g = dloss (exp(s - lse) - onehot),    dx = g W,  dW = g^T x
// Forward: each tile of the product x W^T leaves, per row, the maximum of its logits and the sum of their
// exponentials against it, without the label's; a small kernel joins the tiles to r = log sum_{v != label} exp s_v and
// forms loss = log(1 + exp(r - s_label)).  (As lse - s_label, the difference of near numbers, the loss of a row that the head
// is sure of was what the two were off by: 1e-5 below zero where it is 1e-10.)  Backward:
// the logits of a piece of the vocabulary are formed again, turned into g by the epilogue of the product
// that forms them and kept for the two products that use them.  dx is summed over the pieces in single
// precision, dW of a piece is complete.
// What bounds it: the products, 2 rows hidden vocab operations each (one forward, one to three backward).
//
// This file has the steps around the products, and the products of fp32 operands on the FMA units: 64 x 64
// tiles, 4 x 4 sums a thread.  bf16 goes to the tensor cores (lm_loss_tc.cu).
#include "lm_loss.cuh"

namespace ps {
namespace train {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---- rows that count -----------------------------------------------------------------------------
// One block numbers them, 4096 rows at a time: a running sum of the threads' counts of four rows.
constexpr int kPer = 4;
__global__ void __launch_bounds__(1024) k_loss_rows(int rows, int rows_pad, int V, const int* __restrict__ labels, LossBuf b,
                                                    const float* __restrict__ lse_in, const float* __restrict__ dloss,
                                                    float* loss, float* lse) {
  __shared__ int s_w[2][32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_launch_dependents();
  pdl_wait();
  int base = 0;
  for (int r0 = 0, turn = 0; r0 < rows; r0 += 1024 * kPer, turn ^= 1) {
    const int r = r0 + kPer * tid;
    int lab[kPer], cnt = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) lab[e] = r + e < rows ? labels[r + e] : -1;
#pragma unroll
    for (int e = 0; e < kPer; ++e) cnt += lab[e] >= 0 && lab[e] < V;
    int inc = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) s_w[turn][warp] = inc;
    __syncthreads();                     // (two buffers: the next turn's writers have passed this one's readers)
    int of_warps = s_w[turn][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, of_warps, o);
      if (lane >= o) of_warps += y;
    }
    const int before = __shfl_sync(0xffffffffu, of_warps, warp > 0 ? warp - 1 : 0), all = __shfl_sync(0xffffffffu, of_warps, 31);
    int i = base + (warp > 0 ? before : 0) + inc - cnt;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (r + e >= rows) break;
      const bool counts = lab[e] >= 0 && lab[e] < V;
      b.slot[r + e] = counts ? i : -1;
      if (counts) {
        b.row_of[i] = r + e;
        b.label[i] = lab[e];
        if (lse_in) {
          b.lse[i] = lse_in[r + e];
          b.up[i] = dloss[r + e];
        }
        ++i;
      } else if (loss) {
        loss[r + e] = 0.f;
        lse[r + e] = 0.f;
      }
    }
    base += all;
  }
  if (tid == 0) *b.n = base;
  for (int i = base + tid; i < rows_pad; i += 1024) {   // rows that only fill up a tile
    b.label[i] = -1;
    b.lse[i] = 0.f;
    b.up[i] = 0.f;
  }
}

// Row i of the compact copy from row r of x (r < 0: zeros), by a block of 256 threads.  Forward (with w) also the label's
// logit: the products of the tensor cores truncate as they add (a logit of 1.4 over 5120 terms comes out 1e-5 too near
// zero), which a loss would keep in full while the others' sum averages it.
template <class T>
__device__ __forceinline__ void take_row(int H, int i, int r, int label, const T* __restrict__ x, size_t ldx, const T* __restrict__ w,
                                         const LossBuf& b, bool vec) {
  __shared__ float s_sum[8];
  constexpr int N = 16 / sizeof(T);
  uint4* dst = reinterpret_cast<uint4*>((T*)b.x + (size_t)i * H);
  if (r < 0) {
    for (int c = threadIdx.x; c < H / N; c += 256) dst[c] = make_uint4(0, 0, 0, 0);
    return;
  }
  const T* src = x + (size_t)r * ldx;
  const uint4* row = w ? reinterpret_cast<const uint4*>(w + (size_t)label * H) : nullptr;
  float sum = 0.f;
  for (int c = threadIdx.x; c < H / N; c += 256) {
    uint4 v;
    if (vec) {
      v = reinterpret_cast<const uint4*>(src)[c];
    } else {
      T* e = reinterpret_cast<T*>(&v);
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = src[c * N + j];
    }
    dst[c] = v;
    if (row) {
      const uint4 u = row[c];
      const T *e = reinterpret_cast<const T*>(&v), *f = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < N; ++j) sum = fmaf((float)e[j], (float)f[j], sum);
    }
  }
  if (!row) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 8; ++k) sum += s_sum[k];
    b.picked[i] = sum;
  }
}

// The compact copy behind k_loss_rows, zeros up to the end of the last tile.  A block per row.
template <class T>
__global__ void __launch_bounds__(256) k_loss_gather(int H, int tile, const T* __restrict__ x, size_t ldx, const T* __restrict__ w,
                                                     LossBuf b, bool vec) {
  pdl_launch_dependents();
  pdl_wait();
  const int n = *b.n, i = blockIdx.x;
  if (i >= (n + tile - 1) / tile * tile) return;
  const bool in = i < n;
  take_row<T>(H, i, in ? b.row_of[i] : -1, in ? b.label[i] : -1, x, ldx, w, b, vec);
}

// Both in one launch for few rows: every block counts the labels itself.  The blocks of rows that do not count, and those beyond
// the last row, fill up the tile (there are as many of them as compact rows without a row).
constexpr int kFewRows = 1024;
template <class T>
__global__ void __launch_bounds__(256) k_loss_take(int rows, int H, int tile, int V, const int* __restrict__ labels, const T* __restrict__ x,
                                                   size_t ldx, const T* __restrict__ w, LossBuf b, const float* __restrict__ lse_in,
                                                   const float* __restrict__ dloss, float* loss, float* lse, bool vec) {
  __shared__ int s_cnt[2][8];
  const int tid = threadIdx.x, r = blockIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  int before = 0, n = 0, label = -1;
#pragma unroll
  for (int e = 0; e < kFewRows / 256; ++e) {
    const int k = tid + 256 * e;
    if (k < rows) {
      const int l = labels[k];
      const bool counts = l >= 0 && l < V;
      n += counts;
      before += counts && k < r;
    }
  }
  if (r < rows) label = labels[r];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    n += __shfl_xor_sync(0xffffffffu, n, o);
    before += __shfl_xor_sync(0xffffffffu, before, o);
  }
  if ((tid & 31) == 0) { s_cnt[0][tid >> 5] = n; s_cnt[1][tid >> 5] = before; }
  __syncthreads();
  n = before = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) { n += s_cnt[0][k]; before += s_cnt[1][k]; }
  const bool counts = r < rows && label >= 0 && label < V;
  const int i = counts ? before : n + (r - before);   // (r - before: how many before it do not count)
  if (tid == 0) {
    if (r == 0) *b.n = n;
    if (r < rows) b.slot[r] = counts ? i : -1;
    b.label[i] = counts ? label : -1;
    b.lse[i] = counts && lse_in ? lse_in[r] : 0.f;
    b.up[i] = counts && lse_in ? dloss[r] : 0.f;
    if (counts) b.row_of[i] = r;
    else if (loss && r < rows) loss[r] = lse[r] = 0.f;
  }
  if (i >= (n + tile - 1) / tile * tile) return;
  take_row<T>(H, i, counts ? r : -1, label, x, ldx, w, b, vec);
}

// Joins a row's tiles: a warp per compact row, four tiles a lane in flight.
__global__ void __launch_bounds__(256) k_loss_join(int tiles, LossBuf b, float* loss, float* lse) {
  pdl_wait();
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (i >= *b.n) return;
  const float2* part = b.part + (size_t)i * tiles;
  const float own = b.own[i], picked = b.picked[i];
  const int r = b.row_of[i];
  float m = -INFINITY, s = 0.f;
  bool nan = false;
  for (int t0 = lane; t0 < tiles; t0 += 128) {
    float2 p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = t0 + 32 * e < tiles ? part[t0 + 32 * e] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      nan |= p[e].y != p[e].y;
      if (p[e].x > m) {
        s = s * exp2f((m - p[e].x) * kLog2e) + p[e].y;
        m = p[e].x;
      } else if (p[e].x > -INFINITY) {
        s += p[e].y * exp2f((p[e].x - m) * kLog2e);
      }
    }
  }
  float top = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  s = m > -INFINITY ? s * exp2f((m - top) * kLog2e) : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (__any_sync(0xffffffffu, nan)) s = NAN;
  if (lane < 2) {
    // s has all but the label's logit (vocab = 1: nothing).  Lane 1: lse, that of the logits as the product formed them, which the
    // backward call forms again.  Lane 0: the loss, with the label's logit in single precision.  Both are
    // log(exp x + exp y) = max(x, y) + log(1 + exp(-|x - y|)), the loss with y = 0.
    const float log_s = logf(s), rest = top + log_s, d = lane ? rest - own : (top - picked) + log_s, e = log1pf(expf(-fabsf(d)));
    if (lane) {
      const float high = fmaxf(own, rest);
      lse[r] = high == -INFINITY && own == rest ? high : high + e;
    } else {
      loss[r] = picked == INFINITY ? NAN : (d > 0.f ? d + e : e);     // (inf - inf: no number, like every other logit of +inf)
    }
  }
}

// dx of a row from its sums; a block per row.
template <class T>
__global__ void __launch_bounds__(256) k_loss_dx(int H, int splits, int kb, int pairs, size_t layer, LossBuf b, T* dx, size_t ldx, bool vec) {
  pdl_wait();
  const int i = b.slot[blockIdx.x];
  if (pairs > 0) splits = dx_splits(*b.n, H, kb, pairs);
  T* dst = dx + (size_t)blockIdx.x * ldx;
  const float* a = b.acc + (size_t)(i < 0 ? 0 : i) * H;
  for (int c = 4 * threadIdx.x; c < H; c += 1024) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i >= 0)
      for (int k = 0; k < splits; ++k) {
        const float4 y = *reinterpret_cast<const float4*>(a + k * layer + c);
        s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
      }
    if constexpr (sizeof(T) == 4) {
      if (vec) *reinterpret_cast<float4*>(dst + c) = s;
      else { dst[c] = s.x; dst[c + 1] = s.y; dst[c + 2] = s.z; dst[c + 3] = s.w; }
    } else {
      const __nv_bfloat162 u = __floats2bfloat162_rn(s.x, s.y), v = __floats2bfloat162_rn(s.z, s.w);
      if (vec) {
        *reinterpret_cast<uint2*>(dst + c) = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
      } else {
        dst[c] = u.x; dst[c + 1] = u.y; dst[c + 2] = v.x; dst[c + 3] = v.y;
      }
    }
  }
}

// ---- products on the FMA units ---------------------------------------------------------------------
constexpr int kT = 64, kBK = 32, kPitch = 68;

// TM x 64 tile of A B over k in [k0, k1): 4 TM threads, thread (ty, tx) has rows 4 ty + i and columns 4 tx + j.  TM is 64, or 32
// where tiles of 64 would leave multiprocessors without a block (see few_blocks).  An operand
// is [mn][k] with k contiguous (KC) or [k][mn] with mn contiguous; mn_end: first row (column) that there is none of.  In
// shared memory both are [k][mn], eight columns' place exchanged by k's bits 3 and 4 so that the transposing stores of
// a warp (8 rows of 4 groups of k) fall on 32 banks.
template <bool KC, int TM, class T>
__device__ __forceinline__ void load8(int t, const T* __restrict__ p, size_t ld, int mn0, int mn_end, int k0, int k1, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  constexpr int W = TM / 8;   // threads across the tile's width
  const int mn = KC ? mn0 + t / 4 : mn0 + (t % W) * 8, k = KC ? k0 + (t % 4) * 8 : k0 + t / W;
  const T* q = KC ? p + (size_t)mn * ld + k : p + (size_t)k * ld + mn;
  const int n = KC ? (mn < mn_end ? k1 - k : 0) : (k < k1 ? mn_end - mn : 0);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (n >= 4 * h + 4 && ld % 4 == 0) {
      const float4 x = *reinterpret_cast<const float4*>(q + 4 * h);
      v[4 * h] = x.x; v[4 * h + 1] = x.y; v[4 * h + 2] = x.z; v[4 * h + 3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * h + i < n) v[4 * h + i] = q[4 * h + i];
    }
  }
}
template <bool KC, int TM>
__device__ __forceinline__ void stage8(int t, float* s, const float (&v)[8]) {
  if (KC) {
    const int mn = (t / 4) ^ ((t % 4) * 8), k = (t % 4) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[(k + i) * kPitch + mn] = v[i];
  } else {
    constexpr int W = TM / 8;
    const int k = t / W, mn = ((t % W) * 8) ^ (((k >> 3) & 3) * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float4*>(s + k * kPitch + mn + 4 * h) = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
  }
}
struct TileSmem { float a[kBK * kPitch], b[kBK * kPitch]; };

template <int TM, bool AKC, bool BKC>
__device__ __forceinline__ void tile_product(const float* A, size_t lda, int m0, int m_end, const float* B, size_t ldb, int n0,
                                             int n_end, int k0, int k1, TileSmem& sm, float (&c)[4][4]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) c[i][j] = 0.f;
  // (an operand is [mn][k] in eight values a thread: of A's TM columns of k rows that is one set, of B's 64 one or two)
  constexpr int NB = kT / TM;
  const int t = threadIdx.x;
  float va[8], vb[NB][8];
  auto load = [&](int k) {
    load8<AKC, TM>(t, A, lda, m0, m_end, k, k1, va);
#pragma unroll
    for (int s = 0; s < NB; ++s) load8<BKC, kT>(t + 4 * TM * s, B, ldb, n0, n_end, k, k1, vb[s]);
  };
  load(k0);
  for (int k = k0; k < k1; k += kBK) {
    __syncthreads();
    stage8<AKC, TM>(t, sm.a, va);
#pragma unroll
    for (int s = 0; s < NB; ++s) stage8<BKC, kT>(t + 4 * TM * s, sm.b, vb[s]);
    __syncthreads();
    if (k + kBK < k1) load(k + kBK);
#pragma unroll
    for (int kk = 0; kk < kBK; ++kk) {
      const int sw = ((kk >> 3) & 3) * 8;
      const float4 x = *reinterpret_cast<const float4*>(sm.a + kk * kPitch + ((4 * ty) ^ sw));
      const float4 y = *reinterpret_cast<const float4*>(sm.b + kk * kPitch + ((4 * tx) ^ sw));
      const float xa[4] = {x.x, x.y, x.z, x.w}, yb[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(xa[i], yb[j], c[i][j]);
    }
  }
}

// Logits of a tile -> its rows' maximum and sum (GRAD = false), or g (GRAD = true, vocabulary rows v0 .. v0 + nv).
template <bool GRAD, int TM>
__global__ void __launch_bounds__(4 * TM) k_loss_logits(LossPlan p, LossBuf b, const float* __restrict__ w, int v0, int nv) {
  __shared__ __align__(16) TileSmem sm;
  pdl_launch_dependents();
  pdl_wait();
  const int n = *b.n, m0 = blockIdx.y * TM, n0 = blockIdx.x * kT;
  if (m0 >= n) return;
  float c[4][4];
  tile_product<TM, true, true>((const float*)b.x, p.hidden, m0, n, w + (size_t)v0 * p.hidden, p.hidden, n0, nv, 0, p.hidden, sm, c);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 4 * ty + i;
    const bool in = m < n;
    if (GRAD) {
      const int label = in ? b.label[m] - v0 : -1;
      const float l = in ? b.lse[m] : 0.f, up = in ? b.up[m] : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int v = n0 + 4 * tx + j;
        if (in && v < nv)
          ((float*)b.g)[(size_t)m * p.piece + v] = up * (exp2f((c[i][j] - l) * kLog2e) - (v == label ? 1.f : 0.f));
      }
    } else {
      const int label = in ? b.label[m] : -1;
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int v = n0 + 4 * tx + j;
        if (v == label) {
          b.own[m] = c[i][j];
          c[i][j] = -INFINITY;
        }
        if (v < nv) top = fmaxf(top, c[i][j]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        // (nothing above -inf: no sum, unless a logit is not a number)
        if (n0 + 4 * tx + j < nv && !(c[i][j] == -INFINITY)) s += exp2f((c[i][j] - top) * kLog2e);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (in && tx == 0) b.part[(size_t)m * p.tiles + blockIdx.x] = make_float2(top, s);
    }
  }
}

// dx sums of a piece: rows x hidden, over the piece's vocabulary rows (blockIdx.z: a part of them).
template <int TM>
__global__ void __launch_bounds__(4 * TM) k_loss_dx_tile(LossPlan p, LossBuf b, const float* __restrict__ w, int nv, bool add) {
  __shared__ __align__(16) TileSmem sm;
  pdl_launch_dependents();
  pdl_wait();
  const int n = *b.n, m0 = blockIdx.y * TM, n0 = blockIdx.x * kT;
  if (m0 >= n) return;
  const int per = ((nv + p.splits - 1) / p.splits + 31) / 32 * 32, k0 = min(nv, per * (int)blockIdx.z), k1 = min(nv, k0 + per);
  float c[4][4];
  tile_product<TM, true, false>((const float*)b.g, p.piece, m0, n, w, p.hidden, n0, p.hidden, k0, k1, sm, c);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 4 * ty + i;
    if (m >= n) continue;
    float* a = b.acc + ((size_t)blockIdx.z * p.rows_pad + m) * p.hidden + n0 + 4 * tx;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + 4 * tx + j < p.hidden) a[j] = add ? a[j] + c[i][j] : c[i][j];
  }
}

// dW of a piece: its vocabulary rows x hidden, over the rows.
template <int TM>
__global__ void __launch_bounds__(4 * TM) k_loss_dw_tile(LossPlan p, LossBuf b, float* __restrict__ dw, int nv) {
  __shared__ __align__(16) TileSmem sm;
  pdl_launch_dependents();
  pdl_wait();
  const int m0 = blockIdx.y * TM, n0 = blockIdx.x * kT;
  float c[4][4];
  tile_product<TM, false, false>((const float*)b.g, p.piece, m0, nv, (const float*)b.x, p.hidden, n0, p.hidden, 0, *b.n, sm, c);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 4 * ty + i;
    if (m >= nv) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + 4 * tx + j < p.hidden) dw[(size_t)m * p.hidden + n0 + 4 * tx + j] = c[i][j];
  }
}

// ---- host ------------------------------------------------------------------------------------------
constexpr size_t kPieceBytes = 128u << 20;   // g of a piece

int div_up(int a, int b) { return (a + b - 1) / b; }

LossPlan make_plan(int dtype, int rows, int hidden, int vocab) {
  LossPlan p;
  p.tc = dtype == PS_DTYPE_BF16;
  p.rows = rows; p.hidden = hidden; p.vocab = vocab;
  const int tile_m = p.tc ? 256 : kT;
  p.tile_v = p.tc ? 256 : kT;
  p.rows_pad = div_up(std::max(rows, 1), tile_m) * tile_m;
  p.tiles = p.tc ? 2 * div_up(vocab, p.tile_v) : div_up(vocab, p.tile_v);   // (the tensor cores' tiles in two halves)
  // the vocabulary in pieces of equal size, no more of them than keep g within kPieceBytes (1024 rows at least)
  const size_t per_row = (size_t)p.rows_pad * (p.tc ? 2 : 4);
  const int most = (int)std::max<size_t>(1024, kPieceBytes / per_row / 256 * 256);
  const int pieces = div_up(vocab, most);
  p.piece = div_up(div_up(vocab, pieces), 256) * 256;
  p.splits = p.tc ? kMaxSplits : 1;
  if (!p.tc) {   // enough blocks for dx: its tiles times the parts of a piece
    const int blocks = div_up(rows, kT) * div_up(hidden, kT);
    while (p.splits < 16 && blocks * p.splits < 2 * 148 && p.piece / (2 * p.splits) >= 64) p.splits *= 2;
  }
  return p;
}

LossBuf carve(void* ws, const LossPlan& p, bool backward) {
  Carve c(ws);
  LossBuf b = {};
  b.n = c.take<int>(1);
  b.row_of = c.take<int>(p.rows);
  b.slot = c.take<int>(p.rows);
  b.label = c.take<int>(p.rows_pad);
  b.lse = c.take<float>(p.rows_pad);
  b.up = c.take<float>(p.rows_pad);
  const size_t es = p.tc ? 2 : 4;
  b.x = c.take<char>((size_t)p.rows_pad * p.hidden * es);
  if (!backward) {
    b.part = c.take<float2>((size_t)p.tiles * p.rows_pad);
    b.own = c.take<float>(p.rows_pad);
    b.picked = c.take<float>(p.rows_pad);
  } else {
    b.g = c.take<char>((size_t)p.rows_pad * p.piece * es);
    b.acc = c.take<float>((size_t)p.splits * p.rows_pad * p.hidden);
  }
  b.bytes = c.at;
  return b;
}

bool sizes_ok(int dtype, int rows, int hidden, int vocab) {
  return (dtype == PS_DTYPE_F32 || dtype == PS_DTYPE_BF16) && rows >= 0 && rows <= (1 << 20) && hidden >= 8 &&
         hidden <= 65536 && hidden % 8 == 0 && vocab >= 1 && vocab <= (1 << 20);
}
ps_status check(const Err& err, int dtype, int rows, int hidden, int vocab, const void* w, const void* dw) {
  if (dtype != PS_DTYPE_F32 && dtype != PS_DTYPE_BF16) return err(PS_ERR_INVALID_ARG, "ps_lm_loss: dtype must be 0 or 1");
  if (rows < 0 || rows > (1 << 20) || vocab < 1 || vocab > (1 << 20) || hidden < 1 || hidden > 65536)
    return err(PS_ERR_INVALID_ARG, "ps_lm_loss: 0 <= rows <= 2^20, 1 <= vocab <= 2^20, 1 <= hidden <= 65536");
  if (hidden % 8) return err(PS_ERR_UNSUPPORTED, "ps_lm_loss: hidden must be a multiple of 8");
  if (!aligned(w, 16) || !aligned(dw, 16)) return err(PS_ERR_UNSUPPORTED, "ps_lm_loss: w and dw must lie on a 16-byte boundary");
  return PS_OK;
}

// The rows that count and their compact copy.
template <class T>
cudaError_t launch_rows(const LossArgs& a, const void* x, size_t ldx, const int* labels, const float* lse_in,
                        const float* dloss, float* loss, float* lse, cudaStream_t st) {
  const LossPlan& p = a.p;
  const bool vec = aligned(x, 16) && ldx * sizeof(T) % 16 == 0;
  const int tile = p.tc ? kLossTile : kT;
  const T* w = (const T*)(loss ? a.w : nullptr);
  if (p.rows <= kFewRows)
    return launch_after(k_loss_take<T>, dim3(p.rows_pad), dim3(256), 0, st, true, p.rows, p.hidden, tile, p.vocab, labels, (const T*)x,
                        ldx, w, a.b, lse_in, dloss, loss, lse, vec);
  cudaError_t e = launch_after(k_loss_rows, dim3(1), dim3(1024), 0, st, true, p.rows, p.rows_pad, p.vocab, labels, a.b,
                               lse_in, dloss, loss, lse);
  if (e != cudaSuccess) return e;
  return launch_after(k_loss_gather<T>, dim3(p.rows_pad), dim3(256), 0, st, true, p.hidden, tile, (const T*)x, ldx, w, a.b, vec);
}

// Whether tiles of 64 rows are fewer than multiprocessors: then tiles of 32, whose steps take half as long.  Measured, tiles of 64
// and of 32, us (a call alone in a graph; dx and dw each with the logits' gradient):
//   rows x hidden x vocab   forward      dx            dw            tiles of 64: logits, dx (a part), dw
//   64 x 256 x 1000         16.3 13.7    23.9 20.4     26.3 16.4     16, 4, 64
//   205 x 256 x 1000        32.3 34.2    49.2 43.4     55.6 31.0     64, 16, 64
//   330 x 320 x 1500        38.9 41.6    67.2 61.1     86.1 84.7     144, 30, 120
//   1000 x 320 x 1500       41.4 44.0    106.6 105.5   158 179       384, 80, 120
//   1000 x 768 x 5000       234 252      579 633       492 502       1264, 192, 948
// (forward alone the line is at some 50 tiles; the backward call takes more of a step's time.)
bool few_blocks(int tiles) { return tiles < device_sms(); }

cudaError_t logits_fp32(const LossArgs& a, bool grad, int v0, int nv, cudaStream_t st) {
  const LossPlan& p = a.p;
  const int vt = div_up(nv, kT), mt = div_up(p.rows, kT);
  const float* w = (const float*)a.w;
  if (few_blocks(vt * mt)) {
    const dim3 grid(vt, div_up(p.rows, 32));
    return grad ? launch_after(k_loss_logits<true, 32>, grid, dim3(128), 0, st, true, p, a.b, w, v0, nv)
                : launch_after(k_loss_logits<false, 32>, grid, dim3(128), 0, st, true, p, a.b, w, v0, nv);
  }
  return grad ? launch_after(k_loss_logits<true, 64>, dim3(vt, mt), dim3(256), 0, st, true, p, a.b, w, v0, nv)
              : launch_after(k_loss_logits<false, 64>, dim3(vt, mt), dim3(256), 0, st, true, p, a.b, w, v0, nv);
}

cudaError_t piece_fp32(const LossArgs& a, int v0, int nv, cudaStream_t st) {
  const LossPlan& p = a.p;
  const float* w = (const float*)a.w + (size_t)v0 * p.hidden;
  float* dw = (float*)a.dw + (size_t)v0 * p.hidden;
  const unsigned ht = div_up(p.hidden, kT);
  cudaError_t e = logits_fp32(a, true, v0, nv, st);
  if (e == cudaSuccess && a.want_dx) {
    const int mt = div_up(p.rows, kT);
    if (few_blocks(ht * mt * p.splits))
      e = launch_after(k_loss_dx_tile<32>, dim3(ht, div_up(p.rows, 32), p.splits), dim3(128), 0, st, true, p, a.b, w, nv, v0 > 0);
    else
      e = launch_after(k_loss_dx_tile<64>, dim3(ht, mt, p.splits), dim3(256), 0, st, true, p, a.b, w, nv, v0 > 0);
  }
  if (e == cudaSuccess && a.dw) {
    const int vt = div_up(nv, kT);
    if (few_blocks(ht * vt))
      e = launch_after(k_loss_dw_tile<32>, dim3(ht, div_up(nv, 32)), dim3(128), 0, st, true, p, a.b, dw, nv);
    else
      e = launch_after(k_loss_dw_tile<64>, dim3(ht, vt), dim3(256), 0, st, true, p, a.b, dw, nv);
  }
  return e;
}

}  // namespace
}  // namespace train
}  // namespace ps

using namespace ps;
using namespace ps::train;

extern "C" size_t ps_lm_loss_workspace_bytes(int dtype, int rows, int hidden, int vocab, int backward) {
  if (!sizes_ok(dtype, rows, hidden, vocab)) return 0;
  return carve(nullptr, make_plan(dtype, rows, hidden, vocab), backward != 0).bytes;
}

extern "C" ps_status ps_lm_loss(int dtype, int rows, int hidden, int vocab, const void* x, size_t ldx, const void* w,
                                const int* labels, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                                int* status, char* err_text, size_t err_cap, void* stream) {
  const Err err{err_text, err_cap};
  if (err_text && err_cap) err_text[0] = 0;
  if (ps_status s = check(err, dtype, rows, hidden, vocab, w, nullptr)) return s;
  if (rows == 0) return PS_OK;
  if (!x || !w || !labels || !loss || !lse) return err(PS_ERR_INVALID_ARG, "ps_lm_loss: null pointer");
  if (ldx < (size_t)hidden) return err(PS_ERR_INVALID_ARG, "ps_lm_loss: ldx is smaller than hidden");
  LossArgs a = {};
  a.p = make_plan(dtype, rows, hidden, vocab);
  a.b = carve(workspace, a.p, false);
  if (ps_status s = check_workspace(err, "ps_lm_loss", workspace, workspace_bytes, a.b.bytes)) return s;
  a.w = w;
  a.status = status;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = a.p.tc ? launch_rows<__nv_bfloat16>(a, x, ldx, labels, nullptr, nullptr, loss, lse, st)
                         : launch_rows<float>(a, x, ldx, labels, nullptr, nullptr, loss, lse, st);
  if (e == cudaSuccess) {
    if (a.p.tc) e = loss_forward_tc(a, st);
    else e = logits_fp32(a, false, 0, vocab, st);
  }
  if (e == cudaSuccess)
    e = launch_after(k_loss_join, dim3(div_up(rows, 8)), dim3(256), 0, st, true, a.p.tiles, a.b, loss, lse);
  return err.cuda(e, "ps_lm_loss");
}

extern "C" ps_status ps_lm_loss_backward(int dtype, int rows, int hidden, int vocab, const void* x, size_t ldx,
                                         const void* w, const int* labels, const float* lse, const float* dloss, void* dx,
                                         size_t lddx, void* dw, void* workspace, size_t workspace_bytes, int* status,
                                         char* err_text, size_t err_cap, void* stream) {
  const Err err{err_text, err_cap};
  if (err_text && err_cap) err_text[0] = 0;
  if (ps_status s = check(err, dtype, rows, hidden, vocab, w, dw)) return s;
  if (!dx && !dw) return PS_OK;
  cudaStream_t st = (cudaStream_t)stream;
  const size_t es = dtype == PS_DTYPE_F32 ? 4 : 2;
  if (rows == 0) {
    if (!dw) return PS_OK;
    return err.cuda(cudaMemsetAsync(dw, 0, (size_t)vocab * hidden * es, st), "ps_lm_loss_backward");
  }
  if (!x || !w || !labels || !lse || !dloss) return err(PS_ERR_INVALID_ARG, "ps_lm_loss_backward: null pointer");
  if (ldx < (size_t)hidden || (dx && lddx < (size_t)hidden))
    return err(PS_ERR_INVALID_ARG, "ps_lm_loss_backward: ldx or lddx is smaller than hidden");
  LossArgs a = {};
  a.p = make_plan(dtype, rows, hidden, vocab);
  a.b = carve(workspace, a.p, true);
  if (ps_status s = check_workspace(err, "ps_lm_loss_backward", workspace, workspace_bytes, a.b.bytes)) return s;
  a.w = w; a.dw = dw; a.want_dx = dx != nullptr;
  a.status = status;
  cudaError_t e = a.p.tc ? launch_rows<__nv_bfloat16>(a, x, ldx, labels, lse, dloss, nullptr, nullptr, st)
                         : launch_rows<float>(a, x, ldx, labels, lse, dloss, nullptr, nullptr, st);
  for (int v0 = 0; e == cudaSuccess && v0 < vocab; v0 += a.p.piece) {
    const int nv = std::min(a.p.piece, vocab - v0);
    e = a.p.tc ? loss_piece_tc(a, v0, nv, st) : piece_fp32(a, v0, nv, st);
  }
  if (e == cudaSuccess && dx) {
    const size_t layer = (size_t)a.p.rows_pad * hidden;
    const bool vec = aligned(dx, 16) && lddx * es % 16 == 0;
    if (a.p.tc)
      e = launch_after(k_loss_dx<__nv_bfloat16>, dim3(rows), dim3(256), 0, st, true, hidden, a.p.splits, div_up(a.p.piece, 64),
                       device_sms() / 2, layer, a.b, (__nv_bfloat16*)dx, lddx, vec);
    else
      e = launch_after(k_loss_dx<float>, dim3(rows), dim3(256), 0, st, true, hidden, a.p.splits, 0, 0, layer, a.b, (float*)dx, lddx, vec);
  }
  return err.cuda(e, "ps_lm_loss_backward");
}
