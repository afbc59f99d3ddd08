// Attention under the mask of parallel groups (ps_group_attn, ps_group_attn_backward) on the FMA units: every type,
// stride and alignment.  fp32 runs on these kernels; bf16 on the tensor cores' (group_attn_tc.cu) where pointers and strides
// are multiples of 16 bytes.
//
// 64 query rows x 64 keys a step, 256 threads with 4 x 4 scores each; operands widened to fp32 in shared memory,
// statistics and sums in fp32.  Query tiles hold whole groups, so that the keys of the third kind (a row's own group's
// masks) are the tile's own rows.
//   forward  one pass over the keys with the running maximum and sum of the softmax
//   dq       S and dP = dO V^T again per key tile, dq += dS K
//   dk, dv   a block per key tile and key head goes through the query tiles that see it, of all query heads that
//            share the head: its sums need no other block
// An operand that a row does not see takes no part in its sums (not even times a probability of zero, which
// would carry a value that is not finite over).
#include "group_attn_tc.cuh"

namespace ps {
namespace train {
namespace {

constexpr int kT = 64;
constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <class T>
__device__ __forceinline__ float ld1(const T* p);
template <>
__device__ __forceinline__ float ld1<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ld1<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st1(float* p, float x) { *p = x; }
__device__ __forceinline__ void st1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <int D>
constexpr int kPitch = D + 4;

// Rows [0, n) of a tile to shared memory (zeros behind them); row i is src + (row0 + i step) ld.  Sixteen bytes a load where
// pointer and stride allow it, all of a thread's loads in flight together.
template <class T, int D>
__device__ __forceinline__ void load_tile(float* s, const T* src, size_t ld, size_t row0, int step, int n) {
  constexpr int N = 16 / sizeof(T), kLoads = kT * D / N / kThreads;
  if ((((uintptr_t)src | (ld * sizeof(T))) & 15) == 0) {
    uint4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = threadIdx.x + i * kThreads, r = at / (D / N), c = at % (D / N) * N;
      x[i] = make_uint4(0, 0, 0, 0);
      if (r < n) x[i] = *reinterpret_cast<const uint4*>(src + (row0 + (size_t)r * step) * ld + c);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = threadIdx.x + i * kThreads, r = at / (D / N), c = at % (D / N) * N;
      const T* e = reinterpret_cast<const T*>(&x[i]);
#pragma unroll
      for (int j = 0; j < N; j += 4)
        *reinterpret_cast<float4*>(s + r * kPitch<D> + c + j) = make_float4(ld1(e + j), ld1(e + j + 1), ld1(e + j + 2), ld1(e + j + 3));
    }
    return;
  }
  for (int i = threadIdx.x; i < kT * D; i += kThreads) {
    const int r = i / D, c = i % D;
    s[r * kPitch<D> + c] = r < n ? ld1(src + (row0 + (size_t)r * step) * ld + c) : 0.f;
  }
}
// c[i][j] = A row (ty + 16 i) . B row (tx + 16 j)
template <int D>
__device__ __forceinline__ void dot_tiles(const float* a, const float* b, float (&c)[4][4]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) c[i][j] = 0.f;
#pragma unroll 4
  for (int k = 0; k < D; k += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty + 16 * i) * kPitch<D> + k);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * kPitch<D> + k);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[i][j] = fmaf(x[i].x, y[j].x, c[i][j]);
        c[i][j] = fmaf(x[i].y, y[j].y, c[i][j]);
        c[i][j] = fmaf(x[i].z, y[j].z, c[i][j]);
        c[i][j] = fmaf(x[i].w, y[j].w, c[i][j]);
      }
  }
}
// acc row (ty + 16 i), columns 4 tx + 64 h ..: += sum over c in [lo[i], hi[i]] of p[row][c] b[c][column].
template <int D>
__device__ __forceinline__ void add_product(const float* p, const float* b, const int (&lo)[4], const int (&hi)[4],
                                            float (&acc)[4][D / 16]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  int c0 = kT, c1 = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lo[i] <= hi[i]) { c0 = min(c0, lo[i]); c1 = max(c1, hi[i]); }
  for (int c = c0; c <= c1; ++c) {
    float pr[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pr[i] = p[(ty + 16 * i) * (kT + 1) + c];
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      const float4 y = *reinterpret_cast<const float4*>(b + c * kPitch<D> + 4 * tx + 64 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c < lo[i] || c > hi[i]) continue;
        acc[i][4 * h] = fmaf(pr[i], y.x, acc[i][4 * h]);
        acc[i][4 * h + 1] = fmaf(pr[i], y.y, acc[i][4 * h + 1]);
        acc[i][4 * h + 2] = fmaf(pr[i], y.z, acc[i][4 * h + 2]);
        acc[i][4 * h + 3] = fmaf(pr[i], y.w, acc[i][4 * h + 3]);
      }
    }
  }
}
template <class T, int D>
__device__ __forceinline__ void store_rows(T* dst, size_t ld, size_t row0, int step, int first, int n, const float (&acc)[4][D / 16],
                                           const float (&mul)[4], int period) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty + 16 * i;
    if (r >= n || r % period < first) continue;
    T* d = dst + (row0 + (size_t)r * step) * ld;
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) st1(d + 4 * tx + 64 * h + e, acc[i][4 * h + e] * mul[i]);
  }
}

// A query tile's walk over the key tiles.
struct KeyWalk {
  int ctx, R, n_real, base_rows;   // base_rows: rows of the query tile
  int n_ctx, n_rt, total;          // tiles
  size_t kv0;                      // first context row
  int rho0;                        // the tile's first query row within the sequence
  __device__ KeyWalk(const Seqs& s, int b, int rho0_, int rows) {
    ctx = s.ctx[b]; R = s.R; rho0 = rho0_; base_rows = rows;
    kv0 = s.kv0[b];
    n_real = (rho0 + rows - 1) / R + 1;
    n_ctx = div_up(ctx, kT);
    n_rt = div_up(n_real, kT);
    total = n_ctx + n_rt + (R > 1);
  }
  // Kind, first row, row step and number of keys of tile i, and its first key's index among those of its kind.
  __device__ int tile(int i, size_t& row0, int& step, int& n, int& x0) const {
    if (i < n_ctx) { x0 = i * kT; row0 = kv0 + x0; step = 1; n = min(kT, ctx - x0); return CTX; }
    if (i < n_ctx + n_rt) { x0 = (i - n_ctx) * kT; row0 = kv0 + ctx + (size_t)x0 * R; step = R; n = min(kT, n_real - x0); return REAL; }
    x0 = 0; row0 = kv0 + ctx + rho0; step = 1; n = base_rows; return LOCAL;
  }
  // Columns that query row r of the tile sees.
  __device__ void sees(int kind, int n, int x0, int r, int& lo, int& hi) const {
    lo = 0;
    hi = n - 1;
    if (kind == REAL) hi = min(hi, (rho0 + r) / R - x0);
    if (kind == LOCAL) { lo = r - r % R + 1; hi = r; }
    if (r >= base_rows) hi = -1;
  }
};

__device__ __forceinline__ float red16(float v, bool mx) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, v, o);
    v = mx ? fmaxf(v, y) : v + y;
  }
  return v;
}

template <int D>
constexpr int kTileFloats = kT * kPitch<D>;
constexpr int kPFloats = kT * (kT + 1);

template <class T, int D>
__global__ void __launch_bounds__(kThreads) k_ga_fwd(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(16) float sm[];
  float *sq = sm, *sk = sq + kTileFloats<D>, *sv = sk + kTileFloats<D>, *sp = sv + kTileFloats<D>;
  pdl_launch_dependents();
  pdl_wait();
  const int t = (int)gridDim.x - 1 - (int)blockIdx.x, b = seq_of_tile(s, t), h = blockIdx.y;   // (the longest rows first)
  const int gpt = groups_per_tile(kT, s.R), g0 = (t - s.tile0[b]) * gpt, rows = min(gpt, s.groups[b] - g0) * s.R;
  const KeyWalk w(s, b, g0 * s.R, rows);
  const size_t qrow = (size_t)s.q0[b] + w.rho0;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const T *k = (const T*)a.k + (size_t)(h / a.per) * D, *v = (const T*)a.v + (size_t)(h / a.per) * D;
  load_tile<T, D>(sq, (const T*)a.q + (size_t)h * D, a.ldq, qrow, 1, rows);
  float acc[4][D / 16], top[4], sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    top[i] = -INFINITY;
    sum[i] = 0.f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) acc[i][e] = 0.f;
  }
  for (int x = 0; x < w.total; ++x) {
    size_t row0;
    int step, n, x0, lo[4], hi[4];
    const int kind = w.tile(x, row0, step, n, x0);
    __syncthreads();
    load_tile<T, D>(sk, k, a.ldk, row0, step, n);
    load_tile<T, D>(sv, v, a.ldv, row0, step, n);
    __syncthreads();
    float c[4][4];
    dot_tiles<D>(sq, sk, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w.sees(kind, n, x0, ty + 16 * i, lo[i], hi[i]);
      float m = top[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = tx + 16 * j;
        c[i][j] = col >= lo[i] && col <= hi[i] ? c[i][j] * a.scale : -INFINITY;
        m = fmaxf(m, c[i][j]);
      }
      m = red16(m, true);
      const float ref = m > -INFINITY ? m : 0.f;
      const float old = top[i] > -INFINITY ? exp2f((top[i] - ref) * kLog2e) : 0.f;
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = exp2f((c[i][j] - ref) * kLog2e);
        sp[(ty + 16 * i) * (kT + 1) + tx + 16 * j] = e;
        part += e;
      }
      sum[i] = sum[i] * old + red16(part, false);
      top[i] = m;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) acc[i][e] *= old;
    }
    __syncthreads();
    add_product<D>(sp, sv, lo, hi, acc);
  }
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    inv[i] = 1.f / sum[i];
    if (tx == 0 && ty + 16 * i < rows) a.lse[(size_t)h * a.rows + qrow + ty + 16 * i] = top[i] + logf(sum[i]);
  }
  store_rows<T, D>((T*)a.out + (size_t)h * D, a.ldo, qrow, 1, 0, rows, acc, inv, 1);
}

// delta = dout . out, a warp per (row, head).
template <class T, int D>
__global__ void __launch_bounds__(256) k_ga_delta(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (u >= (long long)a.rows * a.n_heads) return;
  const int r = (int)(u / a.n_heads), h = (int)(u - (long long)r * a.n_heads);
  const T *x = (const T*)a.dout + (size_t)r * a.lddo + (size_t)h * D, *y = (const T*)a.out + (size_t)r * a.ldo + (size_t)h * D;
  float d = 0.f;
  if (sizeof(T) == 2) {
    int lo = 0, hi = s.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s.q0[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int rho = r - s.q0[lo], n = s.ctx[lo] + rho / s.R + 1 + rho % s.R;
    if (n <= kExactKeys) {
      d = delta_of_keys<T, D>(s, a, lo, rho, h, n);
      if (lane == 0) a.delta[(size_t)h * a.rows + r] = d;
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) d = fmaf(ld1(x + lane + 32 * i), ld1(y + lane + 32 * i), d);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
  if (lane == 0) a.delta[(size_t)h * a.rows + r] = d;
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) k_ga_dq(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(16) float sm[];
  float *sq = sm, *so = sq + kTileFloats<D>, *sk = so + kTileFloats<D>, *sv = sk + kTileFloats<D>, *sp = sv + kTileFloats<D>;
  pdl_launch_dependents();
  pdl_wait();
  const int t = (int)gridDim.x - 1 - (int)blockIdx.x, b = seq_of_tile(s, t), h = blockIdx.y;
  const int gpt = groups_per_tile(kT, s.R), g0 = (t - s.tile0[b]) * gpt, rows = min(gpt, s.groups[b] - g0) * s.R;
  const KeyWalk w(s, b, g0 * s.R, rows);
  const size_t qrow = (size_t)s.q0[b] + w.rho0;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const T *k = (const T*)a.k + (size_t)(h / a.per) * D, *v = (const T*)a.v + (size_t)(h / a.per) * D;
  load_tile<T, D>(sq, (const T*)a.q + (size_t)h * D, a.ldq, qrow, 1, rows);
  load_tile<T, D>(so, (const T*)a.dout + (size_t)h * D, a.lddo, qrow, 1, rows);
  float acc[4][D / 16], lse[4], delta[4], one[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty + 16 * i;
    lse[i] = r < rows ? a.lse[(size_t)h * a.rows + qrow + r] : 0.f;
    delta[i] = r < rows ? a.delta[(size_t)h * a.rows + qrow + r] : 0.f;
    one[i] = 1.f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) acc[i][e] = 0.f;
  }
  for (int x = 0; x < w.total; ++x) {
    size_t row0;
    int step, n, x0, lo[4], hi[4];
    const int kind = w.tile(x, row0, step, n, x0);
    __syncthreads();
    load_tile<T, D>(sk, k, a.ldk, row0, step, n);
    load_tile<T, D>(sv, v, a.ldv, row0, step, n);
    __syncthreads();
    float c[4][4], d[4][4];
    dot_tiles<D>(sq, sk, c);
    dot_tiles<D>(so, sv, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w.sees(kind, n, x0, ty + 16 * i, lo[i], hi[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = tx + 16 * j;
        float e = 0.f;
        if (col >= lo[i] && col <= hi[i]) e = exp2f((c[i][j] * a.scale - lse[i]) * kLog2e) * (d[i][j] - delta[i]) * a.scale;
        sp[(ty + 16 * i) * (kT + 1) + col] = e;
      }
    }
    __syncthreads();
    add_product<D>(sp, sk, lo, hi, acc);
  }
  store_rows<T, D>((T*)a.dq + (size_t)h * D, a.lddq, qrow, 1, 0, rows, acc, one, 1);
}

// Key tiles of a sequence: its context, its real rows, and (R > 1) the rows of each query tile, of which the masks
// are stored.
__host__ __device__ inline int key_tiles(int ctx, int groups, int R, int T) {
  return div_up(ctx, T) + div_up(groups, T) + (R > 1 ? div_up(groups, groups_per_tile(T, R)) : 0);
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) k_ga_dkv(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(16) float sm[];
  float *sk = sm, *sv = sk + kTileFloats<D>, *sq = sv + kTileFloats<D>, *so = sq + kTileFloats<D>, *sp = so + kTileFloats<D>,
        *sd = sp + kPFloats, *sl = sd + kPFloats;
  pdl_launch_dependents();
  pdl_wait();
  const int t = blockIdx.x, b = seq_of_tile(s, t), hk = blockIdx.y;
  const int ctx = s.ctx[b], groups = s.groups[b], R = s.R, gpt = groups_per_tile(kT, R);
  const int n_ctx = div_up(ctx, kT), n_rt = div_up(groups, kT);
  int i0 = t - s.tile0[b], kind, n, x0, step = 1, q_begin = 0, q_end = groups * R;
  size_t row0;
  if (i0 < n_ctx) { kind = CTX; x0 = i0 * kT; n = min(kT, ctx - x0); row0 = (size_t)s.kv0[b] + x0; }
  else if (i0 < n_ctx + n_rt) {
    kind = REAL; x0 = (i0 - n_ctx) * kT; n = min(kT, groups - x0); step = R;
    row0 = (size_t)s.kv0[b] + ctx + (size_t)x0 * R;
    q_begin = x0 * R;
  } else {
    kind = LOCAL; x0 = (i0 - n_ctx - n_rt) * gpt * R; n = min(gpt * R, groups * R - x0);
    row0 = (size_t)s.kv0[b] + ctx + x0;
    q_begin = x0; q_end = x0 + n;
  }
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  load_tile<T, D>(sk, (const T*)a.k + (size_t)hk * D, a.ldk, row0, step, n);
  load_tile<T, D>(sv, (const T*)a.v + (size_t)hk * D, a.ldv, row0, step, n);
  float dk[4][D / 16], dv[4][D / 16], one[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    one[i] = 1.f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) dk[i][e] = dv[i][e] = 0.f;
  }
  for (int h = hk * a.per; h < (hk + 1) * a.per; ++h)
    for (int r0 = q_begin; r0 < q_end; r0 += kT) {
      const int rows = min(kT, q_end - r0);
      const size_t qrow = (size_t)s.q0[b] + r0;
      __syncthreads();
      load_tile<T, D>(sq, (const T*)a.q + (size_t)h * D, a.ldq, qrow, 1, rows);
      load_tile<T, D>(so, (const T*)a.dout + (size_t)h * D, a.lddo, qrow, 1, rows);
      if (threadIdx.x < 2 * kT) {
        const int r = threadIdx.x % kT;
        const float* src = threadIdx.x < kT ? a.lse : a.delta;
        sl[threadIdx.x] = r < rows ? src[(size_t)h * a.rows + qrow + r] : 0.f;
      }
      __syncthreads();
      float c[4][4], d[4][4];
      dot_tiles<D>(sk, sq, c);
      dot_tiles<D>(sv, so, d);
      int lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = ty + 16 * i;   // what query columns see this key
        lo[i] = 0;
        hi[i] = rows - 1;
        if (kind == REAL) lo[i] = max(0, (x0 + key) * R - r0);
        if (kind == LOCAL) { lo[i] = key; hi[i] = min(hi[i], key - key % R + R - 1); if (key % R == 0) hi[i] = -1; }
        if (key >= n) hi[i] = -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = tx + 16 * j;
          float p = 0.f, e = 0.f;
          if (col >= lo[i] && col <= hi[i]) {
            p = exp2f((c[i][j] * a.scale - sl[col]) * kLog2e);
            e = p * (d[i][j] - sl[kT + col]) * a.scale;
          }
          sp[key * (kT + 1) + col] = p;
          sd[key * (kT + 1) + col] = e;
        }
      }
      __syncthreads();
      add_product<D>(sp, so, lo, hi, dv);
      add_product<D>(sd, sq, lo, hi, dk);
    }
  const int first = kind == LOCAL ? 1 : 0, period = kind == LOCAL ? R : 1;
  store_rows<T, D>((T*)a.dk + (size_t)hk * D, a.lddk, row0, step, first, n, dk, one, period);
  store_rows<T, D>((T*)a.dv + (size_t)hk * D, a.lddv, row0, step, first, n, dv, one, period);
}

// ---- host ------------------------------------------------------------------------------------------
template <int D>
constexpr int smem_tiles(int tiles, int ps) { return (tiles * kTileFloats<D> + ps * kPFloats + 2 * kT) * 4; }

// Fills in the tiles before each sequence; returns their number.
template <class F>
int number_tiles(Seqs& s, F tiles_of) {
  s.tile0[0] = 0;
  for (int b = 0; b < s.B; ++b) s.tile0[b + 1] = s.tile0[b] + tiles_of(s.ctx[b], s.groups[b]);
  return s.tile0[s.B];
}

template <class T, int D>
cudaError_t forward(Seqs s, const AttnArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int smem = smem_tiles<D>(3, 1);
  if (cudaError_t e = allow_smem((const void*)k_ga_fwd<T, D>, smem, done)) return e;
  const int tiles = number_tiles(s, [&](int, int g) { return div_up(g, groups_per_tile(kT, s.R)); });
  return launch_after(k_ga_fwd<T, D>, dim3(tiles, a.n_heads), dim3(kThreads), smem, st, true, s, a);
}
template <class T, int D>
cudaError_t delta_rows(const Seqs& s, const AttnArgs& a, cudaStream_t st) {
  if (a.rows == 0) return cudaSuccess;
  const long long units = (long long)a.rows * a.n_heads;
  return launch_after(k_ga_delta<T, D>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, true, s, a);
}
template <class T, int D>
cudaError_t backward(Seqs s, const AttnArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done_q{0}, done_kv{0};
  constexpr int smem_q = smem_tiles<D>(4, 1), smem_kv = smem_tiles<D>(4, 2);
  if (cudaError_t e = allow_smem((const void*)k_ga_dq<T, D>, smem_q, done_q)) return e;
  if (cudaError_t e = allow_smem((const void*)k_ga_dkv<T, D>, smem_kv, done_kv)) return e;
  cudaError_t e = cudaSuccess;
  if (a.rows > 0) {
    e = delta_rows<T, D>(s, a, st);
    if (e != cudaSuccess) return e;
    const int tiles = number_tiles(s, [&](int, int g) { return div_up(g, groups_per_tile(kT, s.R)); });
    e = launch_after(k_ga_dq<T, D>, dim3(tiles, a.n_heads), dim3(kThreads), smem_q, st, true, s, a);
    if (e != cudaSuccess) return e;
  }
  const int tiles = number_tiles(s, [&](int c, int g) { return key_tiles(c, g, s.R, kT); });
  if (tiles == 0) return e;
  return launch_after(k_ga_dkv<T, D>, dim3(tiles, a.n_kv), dim3(kThreads), smem_kv, st, true, s, a);
}

// Checks the sizes and fills in the sequences.
ps_status check_sizes(const Err& err, const ps_group_attn_args* a, Seqs* s) {
  if (!a) return err(PS_ERR_INVALID_ARG, "ps_group_attn: null pointer");
  if (a->dtype != PS_DTYPE_F32 && a->dtype != PS_DTYPE_BF16) return err(PS_ERR_INVALID_ARG, "ps_group_attn: dtype must be 0 or 1");
  if (a->B < 1 || a->B > PS_MAX_BATCH) return err(PS_ERR_INVALID_ARG, "ps_group_attn: 1 <= B <= 128");
  if (a->k_masks < 0 || a->k_masks > PS_MAX_MASKS) return err(PS_ERR_INVALID_ARG, "ps_group_attn: 0 <= k_masks <= 15");
  if (a->n_heads < 1 || a->n_heads > 1024 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads)
    return err(PS_ERR_INVALID_ARG, "ps_group_attn: 1 <= n_heads <= 1024, a multiple of n_kv_heads");
  if (a->head_dim != 64 && a->head_dim != 128) return err(PS_ERR_UNSUPPORTED, "ps_group_attn: head_dim must be 64 or 128");
  if (!a->n_ctx || !a->n_groups) return err(PS_ERR_INVALID_ARG, "ps_group_attn: null pointer");
  s->B = a->B;
  s->R = a->k_masks + 1;
  long long q = 0, kv = 0;
  for (int b = 0; b < a->B; ++b) {
    if (a->n_ctx[b] < 0 || a->n_groups[b] < 0) return err(PS_ERR_INVALID_ARG, "ps_group_attn: a size is negative");
    s->ctx[b] = a->n_ctx[b];
    s->groups[b] = a->n_groups[b];
    s->q0[b] = (int)q;
    s->kv0[b] = (int)kv;
    q += (long long)a->n_groups[b] * s->R;
    kv += a->n_ctx[b] + (long long)a->n_groups[b] * s->R;
    if (kv * a->n_heads >= (1ll << 31)) return err(PS_ERR_INVALID_ARG, "ps_group_attn: rows times n_heads must be below 2^31");
  }
  s->q0[a->B] = (int)q;
  s->kv0[a->B] = (int)kv;
  return PS_OK;
}

size_t carve(void* ws, const Seqs& s, const ps_group_attn_args* a, bool backward, AttnArgs* g, TcArgs* t, TcArgs* tk) {
  Carve c(ws);
  const size_t units = (size_t)s.q0[s.B] * a->n_heads;
  if (backward) g->delta = c.take<float>(units);
  if (a->dtype != PS_DTYPE_BF16) return c.at;
  t->gpt = tk->gpt = groups_per_tile(128, s.R);
  t->splits = attn_splits(s, a->n_heads, backward);
  t->none = t->splits > 1 ? 0.f : NAN;
  const size_t parts_q = t->splits > 1 ? units * t->splits * a->head_dim : 0;
  size_t parts_k = 0;
  if (backward) {
    attn_parts(s, a->n_kv_heads, a->n_heads / a->n_kv_heads, tk);
    if (tk->parts > 1) parts_k = (size_t)tk->key_units * 2 * 128 * a->head_dim;
  }
  // (dq's parts are joined before dk and dv are formed)
  t->part_o = tk->part_o = c.take<float>(std::max(parts_q, parts_k));
  t->part_l = c.take<float>(t->splits > 1 && !backward ? units * t->splits : 0);
  if (backward) {
    t->lots = attn_lots(s, a->n_heads);
    g->any = c.take<int>(1);
    t->bad = c.take<uint32_t>((size_t)t->lots * 16 * t->splits);
    t->where = c.take<Where>((size_t)t->lots * 4);
    tk->bad = c.take<uint32_t>((size_t)tk->key_units * 32);
    tk->where = c.take<Where>((size_t)tk->lots * 4);
  }
  return c.at;
}

ps_status run(const ps_group_attn_args* a, bool backward, void* workspace, size_t workspace_bytes, int* status,
              const Err& err, cudaStream_t st) {
  Seqs s;
  if (ps_status e = check_sizes(err, a, &s)) return e;
  const int rows = s.q0[s.B], keys = s.kv0[s.B];
  const size_t wq = (size_t)a->n_heads * a->head_dim, wk = (size_t)a->n_kv_heads * a->head_dim;
  if (!(a->scale - a->scale == 0.f)) return err(PS_ERR_INVALID_ARG, "ps_group_attn: scale must be finite");
  if (a->ldq < wq || a->ldk < wk || a->ldv < wk || a->ldo < wq)
    return err(PS_ERR_INVALID_ARG, "ps_group_attn: a row stride is smaller than its row");
  if (rows && (!a->q || !a->k || !a->v || !a->out || !a->lse)) return err(PS_ERR_INVALID_ARG, "ps_group_attn: null pointer");
  if (backward) {
    if (a->lddo < wq || a->lddq < wq || a->lddk < wk || a->lddv < wk)
      return err(PS_ERR_INVALID_ARG, "ps_group_attn_backward: a row stride is smaller than its row");
    if ((rows && (!a->dout || !a->dq)) || (keys && (!a->dk || !a->dv)))
      return err(PS_ERR_INVALID_ARG, "ps_group_attn_backward: null pointer");
  }
  AttnArgs g = {};
  TcArgs tc = {}, tk = {};
  const size_t need = carve(workspace, s, a, backward, &g, &tc, &tk);
  if (ps_status e = check_workspace(err, "ps_group_attn", workspace, workspace_bytes, need)) return e;
  if (keys == 0 || (!backward && rows == 0)) return PS_OK;
  g.n_heads = a->n_heads; g.n_kv = a->n_kv_heads; g.per = a->n_heads / a->n_kv_heads;
  g.rows = rows; g.scale = a->scale;
  g.q = a->q; g.k = a->k; g.v = a->v; g.ldq = a->ldq; g.ldk = a->ldk; g.ldv = a->ldv;
  g.out = a->out; g.ldo = a->ldo; g.lse = a->lse;
  g.dout = a->dout; g.lddo = a->lddo;
  g.dq = a->dq; g.dk = a->dk; g.dv = a->dv; g.lddq = a->lddq; g.lddk = a->lddk; g.lddv = a->lddv;
  g.status = status;
  const bool f32 = a->dtype == PS_DTYPE_F32, d64 = a->head_dim == 64;
  cudaError_t e;
  if (!f32 && attn_tc_takes(g, backward))
    e = attn_tc(a->head_dim, backward, s, g, tc, tk, st);
  else if (backward)
    e = f32 ? (d64 ? train::backward<float, 64>(s, g, st) : train::backward<float, 128>(s, g, st))
            : (d64 ? train::backward<__nv_bfloat16, 64>(s, g, st) : train::backward<__nv_bfloat16, 128>(s, g, st));
  else
    e = f32 ? (d64 ? forward<float, 64>(s, g, st) : forward<float, 128>(s, g, st))
            : (d64 ? forward<__nv_bfloat16, 64>(s, g, st) : forward<__nv_bfloat16, 128>(s, g, st));
  return err.cuda(e, backward ? "ps_group_attn_backward" : "ps_group_attn");
}

}  // namespace
}  // namespace train
}  // namespace ps

using namespace ps;
using namespace ps::train;

extern "C" size_t ps_group_attn_workspace_bytes(const ps_group_attn_args* a, int backward) {
  Seqs s;
  AttnArgs g = {};
  TcArgs t = {}, tk = {};
  if (check_sizes(Err{nullptr, 0}, a, &s) != PS_OK) return 0;
  return carve(nullptr, s, a, backward != 0, &g, &t, &tk);
}
extern "C" ps_status ps_group_attn(const ps_group_attn_args* a, void* workspace, size_t workspace_bytes, int* status,
                                   char* err_text, size_t err_cap, void* stream) {
  if (err_text && err_cap) err_text[0] = 0;
  return run(a, false, workspace, workspace_bytes, status, Err{err_text, err_cap}, (cudaStream_t)stream);
}
extern "C" ps_status ps_group_attn_backward(const ps_group_attn_args* a, void* workspace, size_t workspace_bytes,
                                            int* status, char* err_text, size_t err_cap, void* stream) {
  if (err_text && err_cap) err_text[0] = 0;
  return run(a, true, workspace, workspace_bytes, status, Err{err_text, err_cap}, (cudaStream_t)stream);
}
