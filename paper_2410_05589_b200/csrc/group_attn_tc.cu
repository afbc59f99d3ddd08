// Attention under the mask of parallel groups on the 5th-generation tensor cores: bf16 operands, fp32 scores, statistics
// and sums.
//
//   forward  S = Q K^T,  P = exp(S - max),  O += P V                 query rows on the 128 lanes
//   dq       S = Q K^T,  dP = dO V^T,  dQ += dS K                    query rows on the lanes
//   dk, dv   S^T = K Q^T,  dP^T = V dO^T,  dV += P^T dO,  dK += dS^T Q   keys on the lanes
// with dS = P (dP - delta).  P and dS are rounded to bf16, the operand type of the products that read them (the sums are
// fp32); they go from registers to tensor memory and are read there as the products' A operand, so that
// shared memory holds nothing but Q, K, V and dO, which tiled TMA brings in the one layout (rows of 64 values,
// 128-byte swizzle) that serves a product over head_dim (K-major) and one over rows (MN-major).
//
// A query tile holds whole groups (128 / R of them), so that the masks of the third kind (see group_attn.cuh) are the
// tile's own rows.  Keys of the second kind lie R rows apart: a map of [group][row of a group][column] fetches
// 128 of them in one box.
//
// dk and dv are sums of one block per key tile over the query tiles, dq one of a block per query tile over the key
// tiles: the scores are formed twice in the backward pass, and no sum depends on the order of atomics.
//
// A product of a probability of zero and a value that is not finite is not zero.  A row of sums that holds
// a value that is not finite is therefore formed again, by one warp, over what the row sees alone.
// Every wait is bounded: on expiry the kernel raises the status word and returns.
#include "group_attn_tc.cuh"
#include "umma_gemm.cuh"

namespace ps {
namespace train {
namespace {

using umma::fence_after_sync;
using umma::fence_before_sync;
using umma::mbar_arrive;
using umma::mbar_arrive_expect_tx;
using umma::mbar_init;
using umma::mbar_wait;
using umma::mma_commit;
using umma::smem_u32;
typedef __nv_bfloat16 bf16;

constexpr int kT = 128;                       // rows of a tile
constexpr int kHalfBytes = kT * 128;          // 64 columns of a tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;                 // a maximum this far (log2) above the reference forces a rescale

template <int D>
constexpr int kTileBytes = kT * D * 2;

// ---- PTX --------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* m, int x, int y, uint64_t* bar) {
  umma::tma_load_2d(dst, m, x, y, bar);
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}
// A in tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(id), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::
          "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
      "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(
          r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ bool all_sync(bool p) { return __all_sync(0xffffffffu, p); }

// Operands in shared memory: a tile is D / 64 halves of 128 rows of 128 bytes (swizzled), 8 rows 1024 bytes.  K-major
// (products over head_dim): step ks of 16 columns.  MN-major (products over rows): step ks of 16 rows.
__device__ __forceinline__ uint64_t desc_k(uint32_t s, int ks) {
  const uint32_t at = s + (ks >> 2) * kHalfBytes + (ks & 3) * 32;
  return (uint64_t)((at & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t s, int ks) {
  const uint32_t at = s + ks * 2048;
  return (uint64_t)((at & 0x3FFFFu) >> 4) | ((uint64_t)(kHalfBytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// fp32 sums, bf16 operands, 128 lanes, n columns; the B operand MN-major or not.
__device__ __forceinline__ constexpr uint32_t idesc(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// d = A B^T over head_dim, both operands from shared memory.
template <int D>
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t a, uint32_t b) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) umma::mma_f16(d, desc_k(a, ks), desc_k(b, ks), idesc(kT, false), ks > 0);
}
// d (+)= A B over 128 rows, A (bf16) in tensor memory: its columns 0..63 and 64..127 at `half` columns' distance.
template <int D>
__device__ __forceinline__ void mma_sums(uint32_t d, uint32_t a, int half, uint32_t b, bool add) {
#pragma unroll
  for (int ks = 0; ks < kT / 16; ++ks)
    mma_ts(d, a + (ks >> 2) * half + (ks & 3) * 8, desc_mn(b, ks), idesc(D, true), add || ks > 0);
}

// ---- tiles ------------------------------------------------------------------------------------------
// A query tile's walk over the key tiles.
struct KeyWalk {
  int ctx, R, n_real, rows, rho0;
  int n_ctx, n_rt, total;
  int kv0, g0;                     // first context row, first group row of the sequence
  __device__ KeyWalk(const Seqs& s, int b, int rho0_, int rows_) {
    ctx = s.ctx[b]; R = s.R; rho0 = rho0_; rows = rows_;
    kv0 = s.kv0[b];
    g0 = kv0 + ctx;
    n_real = (rho0 + rows - 1) / R + 1;
    n_ctx = div_up(ctx, kT);
    n_rt = div_up(n_real, kT);
    total = n_ctx + n_rt + (R > 1);
  }
  // Kind of tile i, its first key's index among those of its kind and their number.
  __device__ int tile(int i, int& x0, int& n) const {
    if (i < n_ctx) { x0 = i * kT; n = min(kT, ctx - x0); return CTX; }
    if (i < n_ctx + n_rt) { x0 = (i - n_ctx) * kT; n = min(kT, n_real - x0); return REAL; }
    x0 = rho0; n = rows; return LOCAL;
  }
  __device__ int key_row(int kind, int x) const { return kind == CTX ? kv0 + x : (kind == REAL ? g0 + x * R : g0 + x); }
  // Columns that query row r of the tile sees (rows that only fill the tile up: all of them).
  __device__ void sees(int kind, int x0, int n, int r, int& lo, int& hi) const {
    lo = 0;
    hi = n - 1;
    if (r >= rows) return;
    if (kind == REAL) hi = min(hi, (rho0 + r) / R - x0);
    if (kind == LOCAL) { lo = r - r % R + 1; hi = r; }
  }
};

// 128 rows of K or V (columns col ..) to shared memory.
template <int D>
__device__ __forceinline__ void load_keys(uint32_t dst, const CUtensorMap* flat, const CUtensorMap* strided, int kind, int row0, int R,
                                          int x0, int col, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, kTileBytes<D>);
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    if (kind == REAL && R > 1) tma_3d(dst + h * kHalfBytes, strided, col + 64 * h, row0 % R, row0 / R + x0, bar);
    else tma_2d(dst + h * kHalfBytes, flat, col + 64 * h, row0 + x0, bar);
  }
}
template <int D>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* flat, int row0, int col, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, kTileBytes<D>);
#pragma unroll
  for (int h = 0; h < D / 64; ++h) tma_2d(dst + h * kHalfBytes, flat, col + 64 * h, row0, bar);
}

template <int N>
__device__ __forceinline__ void store_bf16(bf16* dst, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 8)
    *reinterpret_cast<uint4*>(dst + i) = make_uint4(pack2(x[i], x[i + 1]), pack2(x[i + 2], x[i + 3]), pack2(x[i + 4], x[i + 5]),
                                                    pack2(x[i + 6], x[i + 7]));
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int D>
__device__ __forceinline__ void lane_load(const bf16* p, int lane, float (&x)[D / 32]) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x[i] = __bfloat162float(p[lane + 32 * i]);
}
template <int D>
__device__ __forceinline__ float lane_dot(const float (&x)[D / 32], const float (&y)[D / 32]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) s = fmaf(x[i], y[i], s);
  return warp_sum(s);
}

// The tail of a kernel whose waits are bounded: see umma_gemm.cuh.
__device__ __forceinline__ void finish(int tid, int warp, volatile int* abort_flag, int* status, uint32_t tmem, int cols) {
  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // (copies and MMAs in flight)
    if (tid == 0) atomicOr(status, kStatTimeout);
    __syncthreads();
  }
  if (warp == 1) {
    fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
  }
}
__device__ __forceinline__ void alloc_tmem(uint32_t* where, int cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}

// ---- forward ----------------------------------------------------------------------------------------
// Two blocks an SM, each with one query tile: one's softmax runs beside the other's products.  Warp 0 issues the
// TMA loads, warp 1 the MMAs, warps 2..5 own a row a thread.  S of the next key tile is issued behind O += P V of this
// one (P lies in S's columns: the tensor cores work in order), K and V pass through a ring.
template <int D>
struct Fwd {
  static constexpr int NS = D == 128 ? 2 : 4;
  static constexpr int threads = 192, cols = 256;
  static constexpr int smem = (1 + NS) * kTileBytes<D> + 2048;
};
struct FwdCtl {
  uint64_t full[4], empty[4], q_full, s_full, p_full, o_full;
  uint32_t tmem;
  int abort_flag;
};

// Row r of the tile over the key tiles [i0, i1), by one warp and over the keys it sees alone.
template <int D>
__device__ __noinline__ void fwd_row(const Seqs& s, const AttnArgs& a, const TcArgs& t, const KeyWalk& w, int h, int r, int qrow, int i0,
                                     int i1, int split) {
  const int lane = threadIdx.x & 31;
  const bf16 *k = (const bf16*)a.k + (size_t)(h / a.per) * D, *v = (const bf16*)a.v + (size_t)(h / a.per) * D;
  float q[D / 32], o[D / 32], m = -INFINITY, l = 0.f;
  lane_load<D>((const bf16*)a.q + (size_t)(qrow + r) * a.ldq + (size_t)h * D, lane, q);
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  for (int i = i0; i < i1; ++i) {
    int x0, n, lo, hi;
    const int kind = w.tile(i, x0, n);
    w.sees(kind, x0, n, r, lo, hi);
    for (int c = lo; c <= hi; ++c) {
      const size_t row = w.key_row(kind, x0 + c);
      float x[D / 32], y[D / 32];
      lane_load<D>(k + row * a.ldk, lane, x);
      lane_load<D>(v + row * a.ldv, lane, y);
      const float sc = lane_dot<D>(q, x) * a.scale;
      if (sc > m) {
        const float f = m > -INFINITY ? exp2f((m - sc) * kLog2e) : 0.f;
        l *= f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] *= f;
        m = sc;
      }
      const float p = exp2f((sc - (m > -INFINITY ? m : 0.f)) * kLog2e);
      l += p;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = fmaf(p, y[e], o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l, lse = l == 0.f ? -INFINITY : m + logf(l);
  if (t.splits == 1) {
    bf16* dst = (bf16*)a.out + (size_t)(qrow + r) * a.ldo + (size_t)h * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) dst[lane + 32 * e] = __float2bfloat16_rn(o[e] * inv);
    if (lane == 0) a.lse[(size_t)h * a.rows + qrow + r] = lse;
  } else {
    const size_t at = ((size_t)split * a.n_heads + h) * a.rows + qrow + r;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) t.part_o[at * D + lane + 32 * e] = o[e] * inv;
    if (lane == 0) t.part_l[at] = lse;
  }
}

template <int D>
__global__ void __launch_bounds__(Fwd<D>::threads, 2)
k_gat_fwd(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
          const __grid_constant__ TcArgs t) {
  using F = Fwd<D>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t sq = base, ring = base + kTileBytes<D>;
  FwdCtl& ctl = *reinterpret_cast<FwdCtl*>(smem_raw + (base - raw) + (1 + F::NS) * kTileBytes<D>);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < F::NS; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
    mbar_init(&ctl.q_full, 1);
    mbar_init(&ctl.s_full, 1);
    mbar_init(&ctl.p_full, 4);
    mbar_init(&ctl.o_full, 1);
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_launch_dependents();
  }
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, F::cols);
    fence_before_sync();
  }
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_o = tmem + kT;
  volatile int* abort_flag = &ctl.abort_flag;
  // (the longest rows first, all heads of a tile side by side)
  const int u = (int)(gridDim.x - 1 - blockIdx.x), tile = u / a.n_heads, h = u - tile * a.n_heads, split = blockIdx.y, b = seq_of_tile(s, tile);
  const int gpt = groups_per_tile(kT, s.R), g0 = (tile - s.tile0[b]) * gpt, rows = min(gpt, s.groups[b] - g0) * s.R;
  const KeyWalk w(s, b, g0 * s.R, rows);
  const int qrow = s.q0[b] + w.rho0, i0 = w.total * split / t.splits, i1 = w.total * (split + 1) / t.splits;
  pdl_wait();

  if (warp == 0) {
    if (lane == 0 && i0 < i1) {
      load_rows<D>(sq, &maps.q, qrow, h * D, &ctl.q_full);
      const int col = h / a.per * D;
      int it = 0;
      for (int i = i0; i < i1; ++i) {
        int x0, n;
        const int kind = w.tile(i, x0, n), row0 = kind == CTX ? w.kv0 : w.g0;
        for (int kv = 0; kv < 2; ++kv, ++it) {
          const int slot = it % F::NS;
          if (!mbar_wait(&ctl.empty[slot], ((it / F::NS) & 1) ^ 1, abort_flag)) { i = i1; break; }
          load_keys<D>(ring + slot * kTileBytes<D>, kv ? &maps.v : &maps.k, kv ? &maps.vs : &maps.ks, kind, row0, s.R, x0, col,
                       &ctl.full[slot]);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && i0 < i1) {
      const int n = i1 - i0;
      auto scores = [&](int i) {
        const int it = 2 * i, slot = it % F::NS;
        if (!mbar_wait(&ctl.full[slot], (it / F::NS) & 1, abort_flag)) return false;
        fence_after_sync();
        mma_scores<D>(tmem, sq, ring + slot * kTileBytes<D>);
        mma_commit(&ctl.s_full);
        mma_commit(&ctl.empty[slot]);
        return true;
      };
      bool ok = mbar_wait(&ctl.q_full, 0, abort_flag) && scores(0);
      for (int i = 0; ok && i < n; ++i) {
        const int it = 2 * i + 1, slot = it % F::NS;
        ok = mbar_wait(&ctl.full[slot], (it / F::NS) & 1, abort_flag) && mbar_wait(&ctl.p_full, i & 1, abort_flag);
        if (!ok) break;
        fence_after_sync();
        mma_sums<D>(t_o, tmem, 32, ring + slot * kTileBytes<D>, i > 0);
        mma_commit(&ctl.empty[slot]);
        if (i + 1 < n) ok = scores(i + 1);
        else mma_commit(&ctl.o_full);
      }
    }
  } else {
    const int q = warp & 3, r = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int i = i0; i < i1; ++i) {
      int x0, n, lo, hi;
      const int kind = w.tile(i, x0, n);
      w.sees(kind, x0, n, r, lo, hi);
      ok = all_sync(mbar_wait(&ctl.s_full, (i - i0) & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      uint32_t v[kT];
#pragma unroll
      for (int j = 0; j < kT; j += 32) ld32(tmem + lanes + j, v + j);
      ld_wait();
      if (!all_sync(lo <= 0 && hi >= kT - 1)) {
#pragma unroll
        for (int j = 0; j < kT; ++j)
          if (j < lo || j > hi) v[j] = 0xFF800000u;   // -inf
      }
      float x[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < kT; j += 4)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaxf(x[e], __uint_as_float(v[j + e]));
      const float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      if (i == i0) {
        m = top;
      } else {
        // the sums stay relative to an older maximum until one has grown by 2^kSlack (the products so far are
        // complete: S of this tile was issued behind them)
        const bool grown = (top - m) * c > kSlack;
        if (__any_sync(0xffffffffu, grown)) {
          const float f = grown ? ex2((m - top) * c) : 1.f;
          l *= f;
          if (grown) m = top;
#pragma unroll 1
          for (int j = 0; j < D; j += 32) {
            uint32_t o[32];
            ld32(t_o + lanes + j, o);
            ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            st32(t_o + lanes + j, o);
          }
        }
      }
      const float ref = m > -INFINITY ? m * c : 0.f;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kT; j += 32) {
        uint32_t p[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float y0 = ex2(fmaf(__uint_as_float(v[j + e]), c, -ref)), y1 = ex2(fmaf(__uint_as_float(v[j + e + 1]), c, -ref));
          sum[0] += y0;
          sum[1] += y1;
          p[e / 2] = pack2(y0, y1);
        }
        st16(tmem + lanes + j / 2, p);
      }
      l += sum[0] + sum[1];
      st_wait();
      fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full);
    }
    if (ok && i0 < i1) ok = all_sync(mbar_wait(&ctl.o_full, 0, abort_flag));
    if (ok) {
      fence_after_sync();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const size_t at = t.splits == 1 ? 0 : ((size_t)split * a.n_heads + h) * a.rows + qrow + r;
      bf16* dst = (bf16*)a.out + (size_t)(qrow + r) * a.ldo + (size_t)h * D;
      float odd = l * 0.f;                   // no number once a sum is not finite
#pragma unroll 1
      for (int j = 0; j < D; j += 32) {
        uint32_t o[32];
        float y[32];
        if (i0 < i1) {
          ld32(t_o + lanes + j, o);
          ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          odd = fmaf(__uint_as_float(o[e]), 0.f, odd);
          y[e] = __uint_as_float(o[e]) * inv;
        }
        if (r < rows) {
          if (t.splits == 1) {
            store_bf16<32>(dst + j, y);
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(t.part_o + at * D + j + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
      }
      if (r < rows) {
        const float lse = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
        if (t.splits == 1) a.lse[(size_t)h * a.rows + qrow + r] = lse;
        else t.part_l[at] = lse;
      }
      unsigned bad = __ballot_sync(0xffffffffu, r < rows && odd != 0.f);
      __syncwarp();
      for (; bad; bad &= bad - 1) fwd_row<D>(s, a, t, w, h, 32 * q + __ffs(bad) - 1, qrow, i0, i1, split);
    }
    fence_before_sync();
  }
  finish(tid, warp, abort_flag, a.status, tmem, F::cols);
}

// Joins the parts of a row's keys: a warp per (row, head).
template <int D>
__global__ void __launch_bounds__(256) k_gat_join(const __grid_constant__ AttnArgs a, const __grid_constant__ TcArgs t) {
  pdl_launch_dependents();
  pdl_wait();
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), layer = (long long)a.rows * a.n_heads;
  const int lane = threadIdx.x & 31;
  if (u >= layer) return;
  const int h = (int)(u / a.rows), r = (int)(u - (long long)h * a.rows);
  float top = -INFINITY;
  for (int i = 0; i < t.splits; ++i) top = fmaxf(top, t.part_l[i * layer + u]);
  const float ref = top > -INFINITY ? top : 0.f;
  float o[D / 32], l = 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  for (int i = 0; i < t.splits; ++i) {
    const float x = t.part_l[i * layer + u];
    if (x == -INFINITY) continue;   // (this part has no key that the row sees)
    const float f = exp2f((x - ref) * kLog2e);
    l += f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = fmaf(f, t.part_o[(i * layer + u) * D + lane + 32 * e], o[e]);
  }
  bf16* dst = (bf16*)a.out + (size_t)r * a.ldo + (size_t)h * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dst[lane + 32 * e] = __float2bfloat16_rn(o[e] / l);
  if (lane == 0) a.lse[u] = ref + logf(l);
}

// ---- backward: dq -------------------------------------------------------------------------------------
// One block an SM.  S lies in two buffers and is issued two tiles ahead; dS takes dP's columns, each half of the
// keys (64 columns, one group of four warps) in its own.  While the warps turn dP of a tile into dS, nothing of it is
// behind them in the tensor cores' queue but the next tile's S.
template <int D>
struct Dq {
  static constexpr int NK = 3, NV = 2, threads = 320;
  static constexpr int smem = (2 + NK + NV) * kTileBytes<D> + 2048;
};
struct DqCtl {
  uint64_t k_full[3], k_empty[3], v_full[2], v_empty[2], q_full, s_full[2], dp_full, ds_full, o_full;
  uint32_t tmem;
  int abort_flag;
};

template <int D>
__device__ __noinline__ void dq_row(const AttnArgs& a, const KeyWalk& w, int h, int r, int qrow, int i0, int i1, float* part) {
  const int lane = threadIdx.x & 31;
  const bf16 *k = (const bf16*)a.k + (size_t)(h / a.per) * D, *v = (const bf16*)a.v + (size_t)(h / a.per) * D;
  float q[D / 32], g[D / 32], o[D / 32];
  lane_load<D>((const bf16*)a.q + (size_t)(qrow + r) * a.ldq + (size_t)h * D, lane, q);
  lane_load<D>((const bf16*)a.dout + (size_t)(qrow + r) * a.lddo + (size_t)h * D, lane, g);
  const float lse = a.lse[(size_t)h * a.rows + qrow + r], delta = a.delta[(size_t)h * a.rows + qrow + r];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  for (int i = i0; i < i1; ++i) {
    int x0, n, lo, hi;
    const int kind = w.tile(i, x0, n);
    w.sees(kind, x0, n, r, lo, hi);
    for (int c = lo; c <= hi; ++c) {
      const size_t row = w.key_row(kind, x0 + c);
      float x[D / 32], y[D / 32];
      lane_load<D>(k + row * a.ldk, lane, x);
      lane_load<D>(v + row * a.ldv, lane, y);
      const float p = exp2f((lane_dot<D>(q, x) * a.scale - lse) * kLog2e), ds = p * (lane_dot<D>(g, y) - delta);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = fmaf(ds, x[e], o[e]);
    }
  }
  if (part) {
#pragma unroll
    for (int e = 0; e < D / 32; ++e) part[lane + 32 * e] = o[e] * a.scale;
  } else {
    bf16* dst = (bf16*)a.dq + (size_t)(qrow + r) * a.lddq + (size_t)h * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) dst[lane + 32 * e] = __float2bfloat16_rn(o[e] * a.scale);
  }
}

template <int D>
__global__ void __launch_bounds__(Dq<D>::threads, 1)
k_gat_dq(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
         const __grid_constant__ TcArgs t) {
  using F = Dq<D>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t sq = base, so = sq + kTileBytes<D>, sk = so + kTileBytes<D>, sv = sk + F::NK * kTileBytes<D>;
  DqCtl& ctl = *reinterpret_cast<DqCtl*>(smem_raw + (base - raw) + (2 + F::NK + F::NV) * kTileBytes<D>);
  __shared__ unsigned s_bad[4];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < F::NK; ++i) { mbar_init(&ctl.k_full[i], 1); mbar_init(&ctl.k_empty[i], 1); }
    for (int i = 0; i < F::NV; ++i) { mbar_init(&ctl.v_full[i], 1); mbar_init(&ctl.v_empty[i], 1); }
    mbar_init(&ctl.q_full, 2);
    mbar_init(&ctl.s_full[0], 1);
    mbar_init(&ctl.s_full[1], 1);
    mbar_init(&ctl.dp_full, 1);
    mbar_init(&ctl.ds_full, 8);
    mbar_init(&ctl.o_full, 1);
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_launch_dependents();
  }
  if (tid < 4) s_bad[tid] = 0;
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, 512);
    fence_before_sync();
  }
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_dp = tmem + 2 * kT, t_o = tmem + 3 * kT;
  volatile int* abort_flag = &ctl.abort_flag;
  const int u = (int)(gridDim.x - 1 - blockIdx.x), tile = u / a.n_heads, h = u - tile * a.n_heads, split = blockIdx.y, b = seq_of_tile(s, tile);
  const int gpt = groups_per_tile(kT, s.R), g0 = (tile - s.tile0[b]) * gpt, rows = min(gpt, s.groups[b] - g0) * s.R;
  const KeyWalk w(s, b, g0 * s.R, rows);
  const int qrow = s.q0[b] + w.rho0, i0 = w.total * split / t.splits, i1 = w.total * (split + 1) / t.splits, cnt = i1 - i0;
  pdl_wait();

  if (warp == 0) {
    if (lane == 0 && cnt > 0) {
      load_rows<D>(sq, &maps.q, qrow, h * D, &ctl.q_full);
      load_rows<D>(so, &maps.dout, qrow, h * D, &ctl.q_full);
      const int col = h / a.per * D;
      for (int i = 0; i < cnt; ++i) {
        int x0, n;
        const int kind = w.tile(i0 + i, x0, n), row0 = kind == CTX ? w.kv0 : w.g0, ks = i % F::NK, vs = i % F::NV;
        if (!mbar_wait(&ctl.k_empty[ks], ((i / F::NK) & 1) ^ 1, abort_flag)) break;
        load_keys<D>(sk + ks * kTileBytes<D>, &maps.k, &maps.ks, kind, row0, s.R, x0, col, &ctl.k_full[ks]);
        if (!mbar_wait(&ctl.v_empty[vs], ((i / F::NV) & 1) ^ 1, abort_flag)) break;
        load_keys<D>(sv + vs * kTileBytes<D>, &maps.v, &maps.vs, kind, row0, s.R, x0, col, &ctl.v_full[vs]);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && cnt > 0) {
      auto scores = [&](int i) {
        const int ks = i % F::NK;
        if (!mbar_wait(&ctl.k_full[ks], (i / F::NK) & 1, abort_flag)) return false;
        fence_after_sync();
        mma_scores<D>(tmem + (i & 1) * kT, sq, sk + ks * kTileBytes<D>);
        mma_commit(&ctl.s_full[i & 1]);
        return true;
      };
      auto dprob = [&](int i) {
        const int vs = i % F::NV;
        if (!mbar_wait(&ctl.v_full[vs], (i / F::NV) & 1, abort_flag)) return false;
        fence_after_sync();
        mma_scores<D>(t_dp, so, sv + vs * kTileBytes<D>);
        mma_commit(&ctl.dp_full);
        mma_commit(&ctl.v_empty[vs]);
        return true;
      };
      bool ok = mbar_wait(&ctl.q_full, 0, abort_flag) && scores(0) && dprob(0) && (cnt < 2 || scores(1));
      for (int i = 0; ok && i < cnt; ++i) {
        if (!mbar_wait(&ctl.ds_full, i & 1, abort_flag)) break;
        fence_after_sync();
        const int ks = i % F::NK;
        mma_sums<D>(t_o, t_dp, 64, sk + ks * kTileBytes<D>, i > 0);
        mma_commit(&ctl.k_empty[ks]);
        if (i + 1 < cnt) ok = dprob(i + 1);
        else mma_commit(&ctl.o_full);
        if (ok && i + 2 < cnt) ok = scores(i + 2);
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2, r = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    const float c = a.scale * kLog2e;
    const size_t at = (size_t)h * a.rows + qrow + r;
    const float lse = r < rows ? a.lse[at] * kLog2e : 0.f, delta = r < rows ? a.delta[at] : 0.f;
    bool ok = true;
    for (int i = 0; i < cnt; ++i) {
      int x0, n, lo, hi;
      const int kind = w.tile(i0 + i, x0, n);
      w.sees(kind, x0, n, r, lo, hi);
      lo -= 64 * half;
      hi -= 64 * half;
      ok = all_sync(mbar_wait(&ctl.s_full[i & 1], (i >> 1) & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      uint32_t v[64];
      ld32(tmem + (i & 1) * kT + lanes + 64 * half, v);
      ld32(tmem + (i & 1) * kT + lanes + 64 * half + 32, v + 32);
      ld_wait();
#pragma unroll
      for (int j = 0; j < 64; ++j) v[j] = __float_as_uint(ex2(fmaf(__uint_as_float(v[j]), c, -lse)));
      const bool whole = all_sync(lo <= 0 && hi >= 63);
      ok = all_sync(mbar_wait(&ctl.dp_full, i & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
#pragma unroll
      for (int j = 0; j < 64; j += 32) {
        uint32_t d[32], p[16];
        ld32(t_dp + lanes + 64 * half + j, d);
        ld_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          float x = __uint_as_float(v[j + e]) * (__uint_as_float(d[e]) - delta);
          if (!whole && (j + e < lo || j + e > hi)) x = 0.f;
          d[e] = __float_as_uint(x);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = pack2(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
        st16(t_dp + lanes + 64 * half + j / 2, p);
      }
      st_wait();
      fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.ds_full);
    }
    if (ok && cnt > 0) ok = all_sync(mbar_wait(&ctl.o_full, 0, abort_flag));
    float* part = t.splits == 1 ? nullptr : t.part_o + (((size_t)split * a.n_heads + h) * a.rows + qrow) * D;
    if (ok) {
      fence_after_sync();
      bf16* dst = (bf16*)a.dq + (size_t)(qrow + r) * a.lddq + (size_t)h * D;
      float odd = 0.f;
#pragma unroll
      for (int j = half * (D / 2); j < (half + 1) * (D / 2); j += 32) {
        uint32_t o[32];
        float y[32];
        if (cnt > 0) {
          ld32(t_o + lanes + j, o);
          ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          odd = fmaf(__uint_as_float(o[e]), 0.f, odd);
          y[e] = __uint_as_float(o[e]) * a.scale;
        }
        if (r < rows) {
          if (!part) {
            store_bf16<32>(dst + j, y);
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(part + (size_t)r * D + j + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
      }
      const unsigned bad = __ballot_sync(0xffffffffu, r < rows && odd != 0.f);
      if (lane == 0 && bad) atomicOr(&s_bad[q], bad);
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");   // the eight warps: a row's halves are both stored
    if (ok) {
      unsigned todo = half == 0 ? s_bad[q] : 0u;
      for (; todo; todo &= todo - 1) {
        const int rr = 32 * q + __ffs(todo) - 1;
        dq_row<D>(a, w, h, rr, qrow, i0, i1, part ? part + (size_t)rr * D : nullptr);
      }
    }
    fence_before_sync();
  }
  finish(tid, warp, abort_flag, a.status, tmem, 512);
}

// Adds the parts of dq: a warp per (row, head).
template <int D>
__global__ void __launch_bounds__(256) k_gat_dq_join(const __grid_constant__ AttnArgs a, const __grid_constant__ TcArgs t) {
  pdl_launch_dependents();
  pdl_wait();
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), layer = (long long)a.rows * a.n_heads;
  const int lane = threadIdx.x & 31;
  if (u >= layer) return;
  const int h = (int)(u / a.rows), r = (int)(u - (long long)h * a.rows);
  float o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  for (int i = 0; i < t.splits; ++i)
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] += t.part_o[(i * layer + u) * D + lane + 32 * e];
  bf16* dst = (bf16*)a.dq + (size_t)r * a.lddq + (size_t)h * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dst[lane + 32 * e] = __float2bfloat16_rn(o[e]);
}

// ---- backward: dk, dv -----------------------------------------------------------------------------------
// One block an SM with one key tile; steps over the query tiles of all heads that share the key head.  Tensor memory
// is full with S^T (P^T in its columns), dP^T (dS^T in its columns), dK and dV.  The warps form P^T while the tensor
// cores work on dK and dP^T, and dS^T while they work on dV and the next step's S^T.  A thread owns a key and half of
// the query columns, whose lse and delta a warp of its own puts into shared memory.
template <int D>
struct Dkv {
  static constexpr int NQ = 2, threads = 352;
  static constexpr int smem = (2 + 2 * NQ) * kTileBytes<D> + 1024 + 2 * 2 * kT * 4 + 1024;
};
struct DkvCtl {
  uint64_t q_full[2], q_empty[2], g_full[2], g_empty[2], t_full[2], t_empty[2], k_full, s_full, p_full, dp_full, ds_full, o_full;
  uint32_t tmem;
  int abort_flag;
};

// What a key tile is: its rows and the query rows [q_begin, q_end) of the sequence that see any of it.
struct KeyTile {
  int kind, x0, n, row0, step, q_begin, q_end;
  __device__ KeyTile(const Seqs& s, int b, int i) {
    const int ctx = s.ctx[b], groups = s.groups[b], R = s.R, gpt = groups_per_tile(kT, R);
    const int n_ctx = div_up(ctx, kT), n_rt = div_up(groups, kT), g0 = s.kv0[b] + ctx;
    step = 1;
    q_begin = 0;
    q_end = groups * R;
    if (i < n_ctx) { kind = CTX; x0 = i * kT; n = min(kT, ctx - x0); row0 = s.kv0[b] + x0; }
    else if (i < n_ctx + n_rt) { kind = REAL; x0 = (i - n_ctx) * kT; n = min(kT, groups - x0); step = R; row0 = g0 + x0 * R; q_begin = x0 * R; }
    else { kind = LOCAL; x0 = (i - n_ctx - n_rt) * gpt * R; n = min(gpt * R, groups * R - x0); row0 = g0 + x0; q_begin = x0; q_end = x0 + n; }
  }
  // Query rows (of the sequence) that see key i of the tile: [lo, hi].
  __device__ void seen(int i, int R, int& lo, int& hi) const {
    lo = q_begin;
    hi = q_end - 1;
    if (kind == REAL) lo = (x0 + i) * R;
    if (kind == LOCAL) { lo = x0 + i; hi = x0 + i - i % R + R - 1; if (i % R == 0) hi = -1; }
    if (i >= n) hi = -1;
  }
};

template <int D>
__device__ __noinline__ void dkv_row(const Seqs& s, const AttnArgs& a, const KeyTile& kt, int b, int hk, int i) {
  const int lane = threadIdx.x & 31;
  const size_t row = (size_t)kt.row0 + (size_t)i * kt.step;
  float k[D / 32], v[D / 32], dk[D / 32], dv[D / 32];
  lane_load<D>((const bf16*)a.k + row * a.ldk + (size_t)hk * D, lane, k);
  lane_load<D>((const bf16*)a.v + row * a.ldv + (size_t)hk * D, lane, v);
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dk[e] = dv[e] = 0.f;
  int lo, hi;
  kt.seen(i, s.R, lo, hi);
  for (int h = hk * a.per; h < (hk + 1) * a.per; ++h)
    for (int r = lo; r <= hi; ++r) {
      const size_t qr = (size_t)s.q0[b] + r;
      float x[D / 32], g[D / 32];
      lane_load<D>((const bf16*)a.q + qr * a.ldq + (size_t)h * D, lane, x);
      lane_load<D>((const bf16*)a.dout + qr * a.lddo + (size_t)h * D, lane, g);
      const float p = exp2f((lane_dot<D>(x, k) * a.scale - a.lse[(size_t)h * a.rows + qr]) * kLog2e);
      const float ds = p * (lane_dot<D>(g, v) - a.delta[(size_t)h * a.rows + qr]);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        dv[e] = fmaf(p, g[e], dv[e]);
        dk[e] = fmaf(ds, x[e], dk[e]);
      }
    }
  bf16 *ok = (bf16*)a.dk + row * a.lddk + (size_t)hk * D, *ov = (bf16*)a.dv + row * a.lddv + (size_t)hk * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) {
    ok[lane + 32 * e] = __float2bfloat16_rn(dk[e] * a.scale);
    ov[lane + 32 * e] = __float2bfloat16_rn(dv[e]);
  }
}

template <int D>
__global__ void __launch_bounds__(Dkv<D>::threads, 1)
k_gat_dkv(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  using F = Dkv<D>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t sk = base, sv = sk + kTileBytes<D>, sq = sv + kTileBytes<D>, sg = sq + F::NQ * kTileBytes<D>;
  float* s_stat = reinterpret_cast<float*>(smem_raw + (base - raw) + (2 + 2 * F::NQ) * kTileBytes<D>);   // [slot][lse, delta][128]
  DkvCtl& ctl = *reinterpret_cast<DkvCtl*>(s_stat + 2 * 2 * kT);
  __shared__ unsigned s_bad[4];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.q_full[i], 1); mbar_init(&ctl.q_empty[i], 1);
      mbar_init(&ctl.g_full[i], 1); mbar_init(&ctl.g_empty[i], 1);
      mbar_init(&ctl.t_full[i], 32); mbar_init(&ctl.t_empty[i], 8);
    }
    mbar_init(&ctl.k_full, 2);
    mbar_init(&ctl.s_full, 1);
    mbar_init(&ctl.p_full, 8);
    mbar_init(&ctl.dp_full, 1);
    mbar_init(&ctl.ds_full, 8);
    mbar_init(&ctl.o_full, 1);
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_launch_dependents();
  }
  if (tid < 4) s_bad[tid] = 0;
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, 512);
    fence_before_sync();
  }
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_dp = tmem + kT, t_dk = tmem + 2 * kT, t_dv = tmem + 3 * kT;
  volatile int* abort_flag = &ctl.abort_flag;
  const int tile = blockIdx.x / a.n_kv, hk = blockIdx.x - tile * a.n_kv, b = seq_of_tile(s, tile);
  const KeyTile kt(s, b, tile - s.tile0[b]);
  const int per_head = div_up(kt.q_end - kt.q_begin, kT), cnt = per_head * a.per;
  pdl_wait();

  if (warp == 0) {
    if (lane == 0 && cnt > 0) {
      const int row0 = kt.kind == CTX ? s.kv0[b] : s.kv0[b] + s.ctx[b];
      load_keys<D>(sk, &maps.k, &maps.ks, kt.kind, row0, s.R, kt.x0, hk * D, &ctl.k_full);
      load_keys<D>(sv, &maps.v, &maps.vs, kt.kind, row0, s.R, kt.x0, hk * D, &ctl.k_full);
      for (int i = 0; i < cnt; ++i) {
        const int hh = i / per_head, r0 = s.q0[b] + kt.q_begin + (i - hh * per_head) * kT, col = (hk * a.per + hh) * D, slot = i & 1;
        const uint32_t parity = ((i >> 1) & 1) ^ 1;
        if (!mbar_wait(&ctl.q_empty[slot], parity, abort_flag)) break;
        load_rows<D>(sq + slot * kTileBytes<D>, &maps.q, r0, col, &ctl.q_full[slot]);
        if (!mbar_wait(&ctl.g_empty[slot], parity, abort_flag)) break;
        load_rows<D>(sg + slot * kTileBytes<D>, &maps.dout, r0, col, &ctl.g_full[slot]);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && cnt > 0) {
      auto scores = [&](int i) {
        if (!mbar_wait(&ctl.q_full[i & 1], (i >> 1) & 1, abort_flag)) return false;
        fence_after_sync();
        mma_scores<D>(tmem, sk, sq + (i & 1) * kTileBytes<D>);
        mma_commit(&ctl.s_full);
        return true;
      };
      auto dprob = [&](int i) {
        if (!mbar_wait(&ctl.g_full[i & 1], (i >> 1) & 1, abort_flag)) return false;
        fence_after_sync();
        mma_scores<D>(t_dp, sv, sg + (i & 1) * kTileBytes<D>);
        mma_commit(&ctl.dp_full);
        return true;
      };
      bool ok = mbar_wait(&ctl.k_full, 0, abort_flag) && scores(0) && dprob(0);
      for (int i = 0; ok && i < cnt; ++i) {
        if (!mbar_wait(&ctl.p_full, i & 1, abort_flag)) break;
        fence_after_sync();
        mma_sums<D>(t_dv, tmem, 64, sg + (i & 1) * kTileBytes<D>, i > 0);
        mma_commit(&ctl.g_empty[i & 1]);
        if (i + 1 < cnt && !scores(i + 1)) break;
        if (!mbar_wait(&ctl.ds_full, i & 1, abort_flag)) break;
        fence_after_sync();
        mma_sums<D>(t_dk, t_dp, 64, sq + (i & 1) * kTileBytes<D>, i > 0);
        mma_commit(&ctl.q_empty[i & 1]);
        if (i + 1 < cnt) ok = dprob(i + 1);
        else mma_commit(&ctl.o_full);
      }
    }
  } else if (warp == 2) {
    for (int i = 0; i < cnt; ++i) {
      const int hh = i / per_head, r0 = kt.q_begin + (i - hh * per_head) * kT, slot = i & 1;
      if (!all_sync(mbar_wait(&ctl.t_empty[slot], ((i >> 1) & 1) ^ 1, abort_flag))) break;
      const size_t at = (size_t)(hk * a.per + hh) * a.rows + s.q0[b] + r0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = lane + 32 * e;
        const bool in = r0 + col < kt.q_end;
        s_stat[(2 * slot) * kT + col] = in ? a.lse[at + col] * kLog2e : 0.f;
        s_stat[(2 * slot + 1) * kT + col] = in ? a.delta[at + col] : 0.f;
      }
      mbar_arrive(&ctl.t_full[slot]);
    }
  } else {
    const int q = warp & 3, half = (warp - 3) >> 2, key = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    const float c = a.scale * kLog2e;
    int see0, see1;
    kt.seen(key, s.R, see0, see1);
    bool ok = true;
    for (int i = 0; i < cnt; ++i) {
      const int hh = i / per_head, r0 = kt.q_begin + (i - hh * per_head) * kT + 64 * half, slot = i & 1;
      const int lo = see0 - r0, hi = see1 - r0;
      const bool whole = all_sync(lo <= 0 && hi >= 63);
      const float4 *lse = reinterpret_cast<const float4*>(s_stat + (2 * slot) * kT + 64 * half),
                   *delta = reinterpret_cast<const float4*>(s_stat + (2 * slot + 1) * kT + 64 * half);
      ok = all_sync(mbar_wait(&ctl.t_full[slot], (i >> 1) & 1, abort_flag)) && all_sync(mbar_wait(&ctl.s_full, i & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      uint32_t v[64];
      ld32(tmem + lanes + 64 * half, v);
      ld32(tmem + lanes + 64 * half + 32, v + 32);
      ld_wait();
#pragma unroll
      for (int j = 0; j < 64; j += 4) {
        const float4 y = lse[j / 4];
        const float yy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float p = ex2(fmaf(__uint_as_float(v[j + e]), c, -yy[e]));
          if (!whole && (j + e < lo || j + e > hi)) p = 0.f;
          v[j + e] = __float_as_uint(p);
        }
      }
      {
        uint32_t p[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) p[e] = pack2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
        st32(tmem + lanes + 64 * half, p);
      }
      st_wait();
      fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full);
      ok = all_sync(mbar_wait(&ctl.dp_full, i & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
#pragma unroll
      for (int j = 0; j < 64; j += 32) {
        uint32_t d[32], p[16];
        ld32(t_dp + lanes + 64 * half + j, d);
        ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 y = delta[(j + e) / 4];
          const float yy[4] = {y.x, y.y, y.z, y.w};
          float x[4];
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            x[f] = __uint_as_float(v[j + e + f]) * (__uint_as_float(d[e + f]) - yy[f]);
            if (!whole && (j + e + f < lo || j + e + f > hi)) x[f] = 0.f;
          }
          p[e / 2] = pack2(x[0], x[1]);
          p[e / 2 + 1] = pack2(x[2], x[3]);
        }
        st16(t_dp + lanes + 64 * half + j / 2, p);
      }
      st_wait();
      fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&ctl.ds_full);
        mbar_arrive(&ctl.t_empty[slot]);
      }
    }
    if (ok && cnt > 0) ok = all_sync(mbar_wait(&ctl.o_full, 0, abort_flag));
    if (ok) {
      fence_after_sync();
      const bool mine = key < kt.n && (kt.kind != LOCAL || key % s.R != 0);
      const size_t row = (size_t)kt.row0 + (size_t)key * kt.step;
      bf16 *ok_ = (bf16*)a.dk + row * a.lddk + (size_t)hk * D, *ov = (bf16*)a.dv + row * a.lddv + (size_t)hk * D;
      float odd = 0.f;
#pragma unroll
      for (int j = half * (D / 2); j < (half + 1) * (D / 2); j += 32) {
        uint32_t x[32], z[32];
        float y[32];
        if (cnt > 0) {
          ld32(t_dk + lanes + j, x);
          ld32(t_dv + lanes + j, z);
          ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = z[e] = 0;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          odd = fmaf(__uint_as_float(x[e]), 0.f, odd);
          odd = fmaf(__uint_as_float(z[e]), 0.f, odd);
          y[e] = __uint_as_float(x[e]) * a.scale;
        }
        if (mine) store_bf16<32>(ok_ + j, y);
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(z[e]);
        if (mine) store_bf16<32>(ov + j, y);
      }
      const unsigned bad = __ballot_sync(0xffffffffu, mine && odd != 0.f);
      if (lane == 0 && bad) atomicOr(&s_bad[q], bad);
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (ok) {
      unsigned todo = half == 0 ? s_bad[q] : 0u;
      for (; todo; todo &= todo - 1) dkv_row<D>(s, a, kt, b, hk, 32 * q + __ffs(todo) - 1);
    }
    fence_before_sync();
  }
  finish(tid, warp, abort_flag, a.status, tmem, 512);
}

// ---- host ------------------------------------------------------------------------------------------------
int query_tiles(Seqs& s) {
  s.tile0[0] = 0;
  for (int b = 0; b < s.B; ++b) s.tile0[b + 1] = s.tile0[b] + div_up(s.groups[b], groups_per_tile(kT, s.R));
  return s.tile0[s.B];
}
int key_tiles(Seqs& s) {
  s.tile0[0] = 0;
  for (int b = 0; b < s.B; ++b)
    s.tile0[b + 1] = s.tile0[b] + div_up(s.ctx[b], kT) + div_up(s.groups[b], kT) + (s.R > 1 ? div_up(s.groups[b], groups_per_tile(kT, s.R)) : 0);
  return s.tile0[s.B];
}
// Key tiles of the longest query tile.
int most_keys(const Seqs& s) {
  int n = 0;
  for (int b = 0; b < s.B; ++b)
    if (s.groups[b]) n = std::max(n, div_up(s.ctx[b], kT) + div_up(s.groups[b], kT) + (s.R > 1));
  return n;
}

template <class Kern>
cudaError_t ready(Kern kern, int smem, std::atomic<uint64_t>& done) { return allow_smem((const void*)kern, smem, done); }

template <int D>
cudaError_t forward(const Maps& maps, Seqs s, const AttnArgs& a, const TcArgs& t, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (cudaError_t e = ready(k_gat_fwd<D>, Fwd<D>::smem, done)) return e;
  const int tiles = query_tiles(s);
  cudaError_t e = launch_after(k_gat_fwd<D>, dim3((unsigned)tiles * a.n_heads, t.splits), dim3(Fwd<D>::threads), Fwd<D>::smem, st, true, maps, s, a, t);
  if (e != cudaSuccess || t.splits == 1) return e;
  const long long units = (long long)a.rows * a.n_heads;
  return launch_after(k_gat_join<D>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, true, a, t);
}
template <int D>
cudaError_t backward(const Maps& maps, Seqs s, const AttnArgs& a, const TcArgs& t, cudaStream_t st) {
  static std::atomic<uint64_t> done_q{0}, done_kv{0};
  if (cudaError_t e = ready(k_gat_dq<D>, Dq<D>::smem, done_q)) return e;
  if (cudaError_t e = ready(k_gat_dkv<D>, Dkv<D>::smem, done_kv)) return e;
  cudaError_t e = cudaSuccess;
  if (const int tiles = query_tiles(s)) {
    e = launch_after(k_gat_dq<D>, dim3((unsigned)tiles * a.n_heads, t.splits), dim3(Dq<D>::threads), Dq<D>::smem, st, true, maps, s, a, t);
    if (e == cudaSuccess && t.splits > 1) {
      const long long units = (long long)a.rows * a.n_heads;
      e = launch_after(k_gat_dq_join<D>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, true, a, t);
    }
    if (e != cudaSuccess) return e;
  }
  const int tiles = key_tiles(s);
  return launch_after(k_gat_dkv<D>, dim3((unsigned)tiles * a.n_kv), dim3(Dkv<D>::threads), Dkv<D>::smem, st, true, maps, s, a);
}

}  // namespace

// Parts that a query tile's keys are dealt to, so that few query tiles still fill the device: as many as find room at
// once (two blocks an SM forward, one backward), none with less than two key tiles.
int attn_splits(const Seqs& s, int n_heads, bool backward) {
  Seqs c = s;
  const int blocks = query_tiles(c) * n_heads, room = device_sms() * (backward ? 1 : 2), most = most_keys(s) / 2;
  if (blocks == 0) return 1;
  return std::max(1, std::min(std::min(room / blocks, most), 32));
}

bool attn_tc_takes(const AttnArgs& a, bool backward) {
  auto fits = [](const void* p, size_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld < (1ull << 36); };
  if (!(a.scale >= 0.f)) return false;
  if (!fits(a.q, a.ldq) || !fits(a.k, a.ldk) || !fits(a.v, a.ldv) || !fits(a.out, a.ldo)) return false;
  return !backward || (fits(a.dout, a.lddo) && fits(a.dq, a.lddq) && fits(a.dk, a.lddk) && fits(a.dv, a.lddv));
}

cudaError_t attn_tc(int D, bool backward_, const Seqs& s, const AttnArgs& a, const TcArgs& t, cudaStream_t st) {
  Maps m = {};
  const size_t wq = (size_t)a.n_heads * D, wk = (size_t)a.n_kv * D, keys = s.kv0[s.B];
  bool ok = make_rows_map(&m.q, a.q, a.rows, wq, a.ldq, 1) && make_rows_map(&m.k, a.k, keys, wk, a.ldk, 1) &&
            make_rows_map(&m.v, a.v, keys, wk, a.ldv, 1);
  // (a call with fewer rows than a group has no group)
  if (ok && s.R > 1 && keys >= (size_t)s.R)
    ok = make_rows_map(&m.ks, a.k, keys, wk, a.ldk, s.R) && make_rows_map(&m.vs, a.v, keys, wk, a.ldv, s.R);
  if (ok && backward_) ok = make_rows_map(&m.dout, a.dout, a.rows, wq, a.lddo, 1);
  if (!ok) return cudaErrorNotSupported;
  if (backward_) return D == 64 ? backward<64>(m, s, a, t, st) : backward<128>(m, s, a, t, st);
  return D == 64 ? forward<64>(m, s, a, t, st) : forward<128>(m, s, a, t, st);
}

}  // namespace train
}  // namespace ps
