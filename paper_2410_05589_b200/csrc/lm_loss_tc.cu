// Products of the LM-head loss on the 5th-generation tensor cores (bf16 operands, fp32 sums):
//
//   forward   S = X W^T  -> per row and half tile: maximum and sum of exponentials of all but the label's logit; that one
//   gradient  S = X W^T  -> G = up (exp(S - lse) - onehot), rounded to bf16 (the operand type of the two products
//                           that read it; what they add up is fp32): dx and dw are 2.4e-3 off relatively where
//                           the rounding of the result alone makes it 1.7e-3
//   dx        G W        -> sums over the pieces in fp32, a piece in up to four parts of its k (see dx_splits)
//   dw        G^T X      -> the head's gradient
//
// Two CTAs (one cluster, the two SMs of a TPC) work on a tile of 256 x 256 with tcgen05.mma.cta_group::2: each
// brings 128 rows of either operand into shared memory and holds 128 rows of the sums in its tensor memory, so
// that an operand byte fetched serves 256 sums.  A thread of the epilogue owns a row of the tile: the softmax
// statistics need no exchange between threads.  An operand whose k is contiguous in memory (X and W in S, G in
// dx) is read K-major, one whose k runs over rows (W in dx, G and X in dw) MN-major: nothing is transposed.
//
// Persistent pairs walk the tiles, eight row tiles of a column side by side, so that the pairs that work at one
// time share both operands in L2.  Two accumulators in tensor memory let a tile's epilogue overlap the
// next tile's products.
// What bounds it: the tensor cores, at the clock that the power limit leaves them.  Launches by themselves (cool device):
// logits of 3890 rows, 4096 x 128256, 1.60 PFLOP/s, their gradient 1.63, dW 1.75, dx (sums read and written per piece) 1.44; a
// whole call, forward and backward, 1.23 PFLOP/s of all four products against 1.40 that a library's product alone
// sustains.  Up to 256 rows one tile of rows takes the vocabulary at 6.2 TB/s.  Warp 0 issues the TMA loads, warp 1 the MMAs (of the pair: in the leader CTA), warps
// 2..9 read the sums back.  Every wait is bounded: on expiry the kernel raises the status word and returns.
#include "lm_loss.cuh"
#include "train_status.cuh"
#include "umma_gemm.cuh"

namespace ps {
namespace train {
namespace {

using umma::fence_after_sync;
using umma::fence_before_sync;
using umma::mbar_arrive_expect_tx;
using umma::mbar_init;
using umma::mbar_wait;
using umma::smem_u32;

constexpr int kTile = kLossTile;                 // rows and columns of a pair's tile
constexpr int kBK = 64;                          // k of a stage
constexpr int kOpBytes = 128 * kBK * 2;          // one operand of one CTA
constexpr int kStageBytes = 2 * kOpBytes;
constexpr int kStages = 6;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr uint32_t kPeerMask = 0xFEFFFFFFu;      // shared::cluster address of the same offset in the leader CTA
constexpr int kGroup = 8;                        // row tiles side by side
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = 1048576.f;                // (log2) of a row's maximum
// k blocks (of 64) that a logit is summed over on the tensor cores: longer rows are summed in parts of equal size, which the FMA
// units add.  The tensor cores truncate, and what that takes from a logit is in proportion to it and to the length of the chain:
// lse of 6656 terms came out 1.5e-6 off relatively, in two parts 7.2e-7 (4096 in one: 5.7e-7; parts of 1024: 1.2e-7 to 1.9e-7, for 2
// to 5 % of the product's time).
constexpr int kChain = 64;

enum Mode { FWD, GRAD, DX, DW };

struct Ctl {
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr int kSmem = kStages * kStageBytes + 1024 + (int)sizeof(Ctl);

struct Args {
  LossBuf b;
  int rows_pad, hidden, piece;
  int cols;            // columns of the product that there are: vocabulary rows (FWD, GRAD), features (DX, DW)
  int m_tiles;         // DW: row tiles (vocabulary rows of the piece); else they follow from the rows that count
  int kb;              // k blocks; DW: they follow from the rows that count
  int v0, nv;
  int kb_piece;        // DX: k blocks of a whole piece, which its parts are chosen by
  int tiles;           // FWD: half tiles of a row
  bool add;            // DX: add to what is there
  __nv_bfloat16* dw;   // of the piece
  int* status;
};

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t leader_bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(leader_bar)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(id), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(smem_u32(bar) & kPeerMask) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
  umma::tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
  uint32_t r[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(
          r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// Shared-memory operand of 128 rows (or columns).  K-major: as umma::smem_desc.  MN-major: k rows of 64 values (128
// bytes, swizzled), the second 64 values 64 k rows further on, groups of 8 k rows 1024 bytes apart.
template <bool MN>
__device__ __forceinline__ uint64_t op_desc(uint32_t saddr) {
  const uint64_t lbo = MN ? (kBK * 128) >> 4 : 1;
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (lbo << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Tile number t of m_tiles x n_tiles.
__device__ __forceinline__ void tile_at(int t, int m_tiles, int n_tiles, int& m, int& n) {
  const int per = kGroup * n_tiles, g = t / per, rows = min(kGroup, m_tiles - g * kGroup), i = t - g * per;
  n = i / rows;
  m = g * kGroup + i - n * rows;
}

// A tile of logits in several accumulators, one behind the other: sums a thread's 128 columns of them in its registers and leaves
// the result in the last one; c, the number of the first, becomes that one's.
__device__ __forceinline__ bool add_chains(Ctl& ctl, uint32_t lanes, int chains, int& c, volatile int* abort_flag) {
  float v[128];
#pragma unroll
  for (int j = 0; j < 128; ++j) v[j] = 0.f;
  for (int i = 1;; ++i, ++c) {
    if (!__all_sync(0xffffffffu, mbar_wait(&ctl.acc_full[c & 1], (c >> 1) & 1, abort_flag))) return false;
    fence_after_sync();
#pragma unroll
    for (int j0 = 0; j0 < 128; j0 += 16) {
      const uint32_t at = lanes + (c & 1) * kTile + j0;
      float x[16];
      umma::tmem_ld16(at, x);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j0 + j] += x[j];
      if (i == chains) tmem_st16(at, v + j0);
    }
    if (i == chains) break;
    fence_before_sync();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) arrive_leader(&ctl.acc_empty[c & 1]);
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
  return true;
}

// PARTS: of logits that are summed in several parts.
template <int MODE, bool PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_loss_gemm(const __grid_constant__ CUtensorMap tA, const __grid_constant__ CUtensorMap tB, const __grid_constant__ Args a) {
  constexpr bool A_MN = MODE == DW, B_MN = MODE == DX || MODE == DW;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  Ctl& ctl = *reinterpret_cast<Ctl*>(smem_raw + (base - raw) + kStages * kStageBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&ctl.acc_full[i], 1); mbar_init(&ctl.acc_empty[i], 2 * kEpiWarps); }
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  // (tensor memory is allocated by the pair together: both run first)
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl.tmem_base)), "r"(512)
                 : "memory");
    fence_before_sync();
  }
  cluster_arrive();
  cluster_wait();
  fence_after_sync();
  if (warp == 1) asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  pdl_launch_dependents();   // (with tensor memory in hand: the next kernel's blocks take theirs before they wait for this one)
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem_base;
  volatile int* abort_flag = &ctl.abort_flag;
  pdl_wait();
  const int n = *a.b.n;
  const int m_tiles = MODE == DW ? a.m_tiles : (n + kTile - 1) / kTile, n_tiles = (a.cols + kTile - 1) / kTile;
  const int kb = MODE == DW ? (n + kBK - 1) / kBK : a.kb;
  const int splits = MODE == DX ? dx_splits(n, a.hidden, a.kb_piece, n_pairs) : 1;
  const int tiles = m_tiles * n_tiles * splits;
  const int chains = PARTS ? (kb + kChain - 1) / kChain : 1, parts = MODE == DX ? splits : chains;
  // Tile t: its place, and (dx) its part of the k blocks.
  auto place = [&](int t, int& m, int& nn, int& part) {
    part = MODE == DX ? t / (m_tiles * n_tiles) : 0;
    tile_at(t - part * m_tiles * n_tiles, m_tiles, n_tiles, m, nn);
  };

  if (warp == 0) {
    if (lane == 0) {   // ---- TMA producer
      int st = 0;
      uint32_t parity = 1;
      bool alive = true;
      for (int t = pair; alive && t < tiles; t += n_pairs) {
        int m, nn, part;
        place(t, m, nn, part);
        const int ma = m * kTile + (int)rank * 128, nb = nn * kTile + (int)rank * 128;
        for (int k = kb * part / splits; k < kb * (part + 1) / splits; ++k) {
          if (!mbar_wait(&ctl.empty[st], parity, abort_flag)) { alive = false; break; }
          if (rank == 0) mbar_arrive_expect_tx(&ctl.full[st], 2 * kStageBytes);
          const uint32_t sa = base + st * kStageBytes, sb = sa + kOpBytes, bar = smem_u32(&ctl.full[st]) & kPeerMask;
          if (A_MN) {
            tma_load_pair(sa, &tA, ma, k * kBK, bar);
            tma_load_pair(sa + kOpBytes / 2, &tA, ma + 64, k * kBK, bar);
          } else {
            tma_load_pair(sa, &tA, k * kBK, ma, bar);
          }
          if (B_MN) {
            tma_load_pair(sb, &tB, nb, k * kBK, bar);
            tma_load_pair(sb + kOpBytes / 2, &tB, nb + 64, k * kBK, bar);
          } else {
            tma_load_pair(sb, &tB, k * kBK, nb, bar);
          }
          if (++st == kStages) { st = 0; parity ^= 1; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0 && kb > 0) {   // ---- MMA issuer of the pair
      const uint32_t id = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)A_MN << 15) | ((uint32_t)B_MN << 16) |
                          ((uint32_t)(kTile >> 3) << 17) | (16u << 24);
      int st = 0, c = 0;
      uint32_t parity = 0;
      bool alive = true;
      for (int t = pair; alive && t < tiles; t += n_pairs) {
        int m, nn, part;
        place(t, m, nn, part);
        for (int i = 0; alive && i < chains; ++i, ++c) {
          const int buf = c & 1, at = MODE == DX ? part : i;
          alive = mbar_wait(&ctl.acc_empty[buf], ((c >> 1) & 1) ^ 1, abort_flag);
          if (!alive) break;
          fence_after_sync();
          const uint32_t d = tmem + buf * kTile;
          const int k0 = kb * at / parts, k1 = kb * (at + 1) / parts;
          for (int k = k0; k < k1; ++k) {
            if (!mbar_wait(&ctl.full[st], parity, abort_flag)) { alive = false; break; }
            fence_after_sync();
            const uint32_t sa = base + st * kStageBytes;
            const uint64_t da = op_desc<A_MN>(sa), db = op_desc<B_MN>(sa + kOpBytes);
#pragma unroll
            for (int s = 0; s < kBK / 16; ++s)
              mma_pair(d, da + s * (A_MN ? 128 : 2), db + s * (B_MN ? 128 : 2), id, k > k0 || s > 0);
            commit_pair(&ctl.empty[st]);
            if (++st == kStages) { st = 0; parity ^= 1; }
          }
          if (alive) commit_pair(&ctl.acc_full[buf]);
        }
      }
    }
  } else {
    // ---- epilogue: thread = row of the tile, 128 of its columns
    const int q = warp & 3, half = (warp - 2) >> 2, r = 32 * q + lane;
    int c = 0;
    for (int t = pair; t < tiles; t += n_pairs, ++c) {
      int mt, nt, part;
      place(t, mt, nt, part);
      const int m = mt * kTile + (int)rank * 128 + r, c0 = nt * kTile + half * 128;
      const int own = MODE == FWD ? a.b.label[m] - c0 : -1;   // the label's column of these 128
      const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16) + half * 128;
      if (PARTS && !add_chains(ctl, lanes, chains, c, abort_flag)) break;
      const int buf = c & 1;
      const bool ok = PARTS || kb == 0 || mbar_wait(&ctl.acc_full[buf], (c >> 1) & 1, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) break;
      fence_after_sync();
      const uint32_t ta = lanes + buf * kTile;
      if (MODE == FWD) {
        float top = -INFINITY, sum = 0.f;
#pragma unroll 1
        for (int j0 = 0; j0 < 128; j0 += 32) {
          float v[32];
          tmem_ld32(ta + j0, v);
          const int left = a.cols - c0 - j0;
          float mx = top;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (j >= left) v[j] = -INFINITY;
            mx = fmaxf(mx, v[j]);
          }
          float l = mx > -INFINITY ? mx * kLog2e : 0.f;   // (nothing above -inf: the sum stays 0, or no number)
          const bool here = own >= j0 && own < j0 + 32;
          if (__any_sync(0xffffffffu, here || fabsf(l) > kFar)) {
            float x = 0.f;
            mx = top;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (j0 + j == own) {
                x = v[j];
                v[j] = -INFINITY;
              }
              mx = fmaxf(mx, v[j]);
            }
            if (here) a.b.own[m] = x;
            // (v log2(e) - l is what l's rounding left where the two are equal: beyond single precision's exponents from 2^31 on)
            const bool far = fabsf(mx > -INFINITY ? mx * kLog2e : 0.f) > kFar;
            l = mx > -INFINITY && !far ? mx * kLog2e : 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (far) v[j] -= mx;
          }
          sum *= top > -INFINITY ? exp2f((top - mx) * kLog2e) : 0.f;
          top = mx;
          float s0 = 0.f, s1 = 0.f;
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            s0 += exp2f(fmaf(v[j], kLog2e, -l));
            s1 += exp2f(fmaf(v[j + 1], kLog2e, -l));
          }
          sum += s0 + s1;
        }
        if (m < n) a.b.part[(size_t)m * a.tiles + 2 * nt + half] = make_float2(top, sum);
      } else if (MODE == GRAD) {
        const bool in = m < n;
        const float l = a.b.lse[m] * kLog2e, up = a.b.up[m];
        const int label = a.b.label[m] - a.v0;
        uint4* dst = reinterpret_cast<uint4*>((__nv_bfloat16*)a.b.g + (size_t)m * a.piece + c0);
#pragma unroll 1
        for (int j0 = 0; j0 < 128; j0 += 32) {
          float v[32];
          tmem_ld32(ta + j0, v);
          const int left = a.nv - c0 - j0, at = label - c0 - j0;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float e = exp2f(fmaf(v[j], kLog2e, -l)) - (j == at ? 1.f : 0.f);
            v[j] = in && j < left ? up * e : 0.f;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 8)
            dst[(j0 + j) / 8] = make_uint4(pack2(v[j], v[j + 1]), pack2(v[j + 2], v[j + 3]), pack2(v[j + 4], v[j + 5]),
                                           pack2(v[j + 6], v[j + 7]));
        }
      } else if (MODE == DX) {
        const bool none = kb * part / splits == kb * (part + 1) / splits;   // (fewer k blocks than parts)
        float* dst = a.b.acc + ((size_t)part * a.rows_pad + m) * a.hidden;
#pragma unroll 1
        for (int j0 = 0; j0 < 128; j0 += 32) {
          float v[32];
          tmem_ld32(ta + j0, v);
          if (none) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
          }
          if (m < n) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const int col = c0 + j0 + j;
              if (col < a.hidden) {
                float4 x = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                float4* d = reinterpret_cast<float4*>(dst + col);
                if (a.add) {
                  const float4 y = *d;
                  x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                }
                *d = x;
              }
            }
          }
        }
      } else {
        __nv_bfloat16* dst = a.dw + (size_t)m * a.hidden;
#pragma unroll 1
        for (int j0 = 0; j0 < 128; j0 += 32) {
          float v[32];
          if (kb > 0) tmem_ld32(ta + j0, v);
          else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
          }
          if (m < a.nv) {
#pragma unroll
            for (int j = 0; j < 32; j += 8)
              if (c0 + j0 + j < a.hidden)
                *reinterpret_cast<uint4*>(dst + c0 + j0 + j) = make_uint4(
                    pack2(v[j], v[j + 1]), pack2(v[j + 2], v[j + 3]), pack2(v[j + 4], v[j + 5]), pack2(v[j + 6], v[j + 7]));
          }
        }
      }
      fence_before_sync();
      __syncwarp();
      if (lane == 0) arrive_leader(&ctl.acc_empty[buf]);
    }
    fence_before_sync();
  }

  __syncthreads();
  if (ctl.abort_flag) {
    // let copies and MMAs that are still in flight finish before shared and tensor memory go
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    if (tid == 0) report_timeout(a.status);
    __syncthreads();
  }
  cluster_arrive();
  cluster_wait();   // neither CTA leaves while the other's copies, MMAs or arrivals may still touch it
  if (warp == 1) {
    fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <int MODE, bool PARTS>
cudaError_t launch_as(const CUtensorMap& tA, const CUtensorMap& tB, const Args& g, int most_tiles, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem((const void*)k_loss_gemm<MODE, PARTS>, kSmem, done);
  if (e != cudaSuccess) return e;
  const int pairs = std::min(most_tiles, device_sms() / 2);
  return launch_after(k_loss_gemm<MODE, PARTS>, dim3(2 * pairs), dim3(kThreads), kSmem, st, true, tA, tB, g);
}
template <int MODE>
cudaError_t launch(const CUtensorMap& tA, const CUtensorMap& tB, const Args& g, int most_tiles, cudaStream_t st) {
  // (two kernels: the sums of several parts take 168 registers a thread, with which a block does not start beside those of the
  // kernel before it: 2 us of a call)
  if constexpr (MODE == FWD || MODE == GRAD)
    if (g.kb > kChain) return launch_as<MODE, true>(tA, tB, g, most_tiles, st);
  return launch_as<MODE, false>(tA, tB, g, most_tiles, st);
}

Args common(const LossArgs& a) {
  Args g = {};
  g.b = a.b;
  g.rows_pad = a.p.rows_pad; g.hidden = a.p.hidden; g.piece = a.p.piece;
  g.status = a.status;
  return g;
}

}  // namespace

cudaError_t loss_forward_tc(const LossArgs& a, cudaStream_t st) {
  const LossPlan& p = a.p;
  CUtensorMap x, w;
  if (!make_map(&x, a.b.x, p.rows_pad, p.hidden, 128) || !make_map(&w, a.w, p.vocab, p.hidden, 128)) return cudaErrorNotSupported;
  Args g = common(a);
  g.cols = p.vocab;
  g.kb = (p.hidden + kBK - 1) / kBK;
  g.tiles = p.tiles;
  return launch<FWD>(x, w, g, p.rows_pad / kTile * ((p.vocab + kTile - 1) / kTile), st);
}

cudaError_t loss_piece_tc(const LossArgs& a, int v0, int nv, cudaStream_t st) {
  const LossPlan& p = a.p;
  const __nv_bfloat16* w = (const __nv_bfloat16*)a.w + (size_t)v0 * p.hidden;
  const int mt = p.rows_pad / kTile, vt = (nv + kTile - 1) / kTile, ht = (p.hidden + kTile - 1) / kTile;
  CUtensorMap xk, wk;
  if (!make_map(&xk, a.b.x, p.rows_pad, p.hidden, 128) || !make_map(&wk, w, nv, p.hidden, 128)) return cudaErrorNotSupported;
  Args g = common(a);
  g.v0 = v0; g.nv = nv;
  g.cols = nv;
  g.kb = (p.hidden + kBK - 1) / kBK;
  cudaError_t e = launch<GRAD>(xk, wk, g, mt * vt, st);
  if (e == cudaSuccess && a.want_dx) {
    CUtensorMap gk, wm;
    if (!make_map(&gk, a.b.g, p.rows_pad, p.piece, 128) || !make_map(&wm, w, nv, p.hidden, 64)) return cudaErrorNotSupported;
    g.cols = p.hidden;
    g.kb = (nv + kBK - 1) / kBK;
    g.kb_piece = (p.piece + kBK - 1) / kBK;
    g.add = v0 > 0;
    e = launch<DX>(gk, wm, g, device_sms() / 2, st);   // (the parts depend on the rows that count and on the number of pairs)
  }
  if (e == cudaSuccess && a.dw) {
    CUtensorMap gm, xm;
    if (!make_map(&gm, a.b.g, p.rows_pad, p.piece, 64) || !make_map(&xm, a.b.x, p.rows_pad, p.hidden, 64)) return cudaErrorNotSupported;
    g.cols = p.hidden;
    g.m_tiles = vt;
    g.dw = (__nv_bfloat16*)a.dw + (size_t)v0 * p.hidden;
    e = launch<DW>(gm, xm, g, vt * ht, st);
  }
  return e;
}

cudaError_t loss_take_status(int* word, cudaStream_t st) { return take_word(word, st); }
cudaError_t loss_wait_expires(long long limit, int* status, cudaStream_t st) { return wait_expires(limit, status, st); }

}  // namespace train
}  // namespace ps
