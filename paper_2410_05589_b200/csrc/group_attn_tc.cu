// Attention under the mask of parallel groups on the 5th-generation tensor cores: bf16 operands, fp32 scores, statistics
// and sums.
//
//   forward  S = Q K^T,  P = exp(S - max),  O += P V                 query rows on the 128 lanes
//   dq       S = Q K^T,  dP = dO V^T,  dQ += dS K                    query rows on the lanes
//   dk, dv   S^T = K Q^T,  dP^T = V dO^T,  dV += P^T dO,  dK += dS^T Q   keys on the lanes (masks: see k_gat_masks)
// with dS = P (dP - delta).  P and dS are rounded to bf16, the operand type of the products that read them (an MMA has both
// operands of one type, and V, K, Q and dO are bf16; a second, low half of P would be half as many products again).  The sums are
// fp32: out and the gradients are 2.3e-3 off where the rounding of the result alone makes it 1.7e-3.  They go from registers to tensor memory and are read there as the products' A operand, so that
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
// a value that is not finite is therefore formed again, by one warp, over what the row sees alone: in the forward kernel by the
// block that has it, behind its last wait; in the backward pass by a kernel of its own (k_gat_again), since the persistent
// blocks' next units wait, within bounds, for the warps that would do it.
// Every wait is bounded: on expiry the kernel raises the status word and returns.
#include "group_attn_tc.cuh"
#include "train_status.cuh"
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
constexpr float kFar = 1048576.f;             // (log2) of a reference: see the forward kernel
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
__device__ __forceinline__ void ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
template <int N>
__device__ __forceinline__ void ldn(uint32_t taddr, uint32_t* r) {
  if constexpr (N == 32) ld32(taddr, r); else ld16(taddr, r);
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(
          r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
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
__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
  return m;
}
// Two fp32 operations an instruction.
struct f2 { float x, y; };
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 d;
  asm("{\n\t.reg .b64 p, q, r, s;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%6, %7};\n\t"
      "fma.rn.f32x2 s, p, q, r;\n\tmov.b64 {%0, %1}, s;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 d;
  asm("{\n\t.reg .b64 p, q, s;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\t"
      "add.rn.f32x2 s, p, q;\n\tmov.b64 {%0, %1}, s;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 d;
  asm("{\n\t.reg .b64 p, q, s;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\t"
      "mul.rn.f32x2 s, p, q;\n\tmov.b64 {%0, %1}, s;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ f2 pair_of(const uint32_t* v) { return f2{__uint_as_float(v[0]), __uint_as_float(v[1])}; }
__device__ __forceinline__ bool all_sync(bool p) { return __all_sync(0xffffffffu, p); }

// Operands in shared memory: a tile is D / 64 halves of 128 rows of 128 bytes (swizzled), 8 rows 1024 bytes.  K-major
// (products over head_dim) or MN-major (products over rows: 64 columns, then the other half); what a step of 16 columns or 16
// rows adds is a constant, since the issuing thread's instructions between two products are time the tensor cores wait.
__device__ __forceinline__ uint64_t desc_k(uint32_t s) {
  return (uint64_t)((s & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t s) {
  return (uint64_t)((s & 0x3FFFFu) >> 4) | ((uint64_t)(kHalfBytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
__host__ __device__ constexpr int step_k(int ks) { return ((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4; }
__host__ __device__ constexpr int step_mn(int ks) { return ks * 2048 >> 4; }
// fp32 sums, bf16 operands, 128 lanes, n columns; the B operand MN-major or not.
__device__ __forceinline__ constexpr uint32_t idesc(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// d = A B^T over head_dim, both operands from shared memory.
template <int D>
__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) umma::mma_f16(d, a + step_k(ks), b + step_k(ks), idesc(kT, false), ks > 0);
}
// d (+)= A B over 128 rows, A (bf16) in tensor memory: the columns of W rows lie together, at W columns' distance (a thread
// stores what it forms of W fp32 columns in the first half of the same).
template <int D, int W>
__device__ __forceinline__ void mma_sums(uint32_t d, uint32_t a, uint64_t b, bool add) {
#pragma unroll
  for (int ks = 0; ks < kT / 16; ++ks)
    mma_ts(d, a + ks * 16 / W * W + ks * 16 % W / 2, b + step_mn(ks), idesc(D, true), add || ks > 0);
}

// What the rows of a warp see of columns j .. j + 31.
enum { kNone, kSome, kAll };
__device__ __forceinline__ int chunk_sees(int j, int lo, int hi) {
  if (all_sync(lo <= j && hi >= j + 31)) return kAll;
  return all_sync(hi < j || lo > j + 31) ? kNone : kSome;
}
// One bit for each of them that this row sees.
__device__ __forceinline__ uint32_t seen_bits(int j, int lo, int hi) {
  const uint32_t below = hi < j ? 0u : (hi >= j + 31 ? ~0u : (2u << (hi - j)) - 1);
  return lo <= j ? below : (lo > j + 31 ? 0u : below & (~0u << (lo - j)));
}
// Their scores: -inf where it does not; products with them: zero.
__device__ __forceinline__ void mask_scores(uint32_t* w, int j, int lo, int hi) {
  const uint32_t bits = seen_bits(j, lo, hi);
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!(bits & (1u << e))) w[e] = 0xFF800000u;
}
__device__ __forceinline__ void mask_zero(uint32_t* w, int j, int lo, int hi) {
  const uint32_t bits = seen_bits(j, lo, hi);
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!(bits & (1u << e))) w[e] = 0;
}

// ---- tiles ------------------------------------------------------------------------------------------
// Key tiles that a query tile of a sequence goes through, in order: the context, the real rows up to those of its last
// group, then (R > 1) its own rows.
struct KeyWalk {
  int ctx, R, n_real;              // n_real: groups up to the last of the query tile
  int n_ctx, n_shared, total;
  int kv0, g0;                     // first context row, first group row of the sequence
  __device__ void start(const Seqs& s, int b, int group_end) {
    ctx = s.ctx[b]; R = s.R; n_real = group_end;
    kv0 = s.kv0[b];
    g0 = kv0 + ctx;
    n_ctx = div_up(ctx, kT);
    n_shared = n_ctx + div_up(n_real, kT);
    total = n_shared + (R > 1);
  }
  // Kind of tile i, its first key's index among those of its kind and their number; the query tile begins with group
  // `group` and has n_rows.
  __device__ int tile(int i, int group, int n_rows, int& x0, int& n) const {
    if (i < n_ctx) { x0 = i * kT; n = min(kT, ctx - x0); return CTX; }
    if (i < n_shared) { x0 = (i - n_ctx) * kT; n = min(kT, n_real - x0); return REAL; }
    x0 = group * R; n = n_rows; return LOCAL;
  }
  __device__ int key_row(int kind, int x) const { return kind == CTX ? kv0 + x : (kind == REAL ? g0 + x * R : g0 + x); }
};
// Row r of a query tile: its group within the tile and its place in the group.
struct TileRow {
  int r, group, place;
  __device__ TileRow(int r_, int R) : r(r_), group(r_ / R), place(r_ - r_ / R * R) {}
  // Columns of a key tile that it sees (rows that only fill the query tile up: all of them).
  __device__ void sees(int kind, int x0, int n, int first_group, int n_rows, int& lo, int& hi) const {
    lo = 0;
    hi = n - 1;
    if (r >= n_rows) return;
    if (kind == REAL) hi = min(hi, first_group + group - x0);
    if (kind == LOCAL) { lo = r - place + 1; hi = r; }
  }
};

// One unit of work of the kernels whose lanes are query rows: a query tile of a head and a part of its key tiles.  (It
// goes by value, to stay in registers: as an object in memory it was read again behind every instruction that may touch
// memory.)
struct QueryWork {
  int b, h, split, group, rows, qrow, i0, i1;   // first group, rows, first row of the tile; key tiles [i0, i1)
  KeyWalk w;
  __device__ static int count(const Seqs& s, const AttnArgs& a, const TcArgs& t) { return s.tile0[s.B] * a.n_heads * t.splits; }
  // (unit 0 is the last one: the longest rows of the longest sequence)
  __device__ QueryWork(const Seqs& s, const AttnArgs& a, const TcArgs& t, int unit) {
    int u = count(s, a, t) - 1 - unit;
    split = 0;
    if (t.splits > 1) { split = u % t.splits; u /= t.splits; }
    const int tile = u / a.n_heads;
    h = u - tile * a.n_heads;
    b = seq_of_tile(s, tile);
    group = (tile - s.tile0[b]) * t.gpt;
    const int n = min(t.gpt, s.groups[b] - group);
    rows = n * s.R;
    qrow = s.q0[b] + group * s.R;
    w.start(s, b, group + n);
    i0 = 0;
    i1 = w.total;
    if (t.splits > 1) {
      i0 = w.total * split / t.splits;
      i1 = w.total * (split + 1) / t.splits;
    }
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
// C = D / 32 neighbouring channels of a row, bf16: a lane's part of it.
template <int C>
struct Chans { uint32_t v[C / 2]; };
template <int C>
__device__ __forceinline__ Chans<C> chan_load(const bf16* p) {
  Chans<C> r;
  if constexpr (C == 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    r.v[0] = x.x; r.v[1] = x.y; r.v[2] = x.z; r.v[3] = x.w;
  } else if constexpr (C == 4) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    r.v[0] = x.x; r.v[1] = x.y;
  } else {
    r.v[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  return r;
}
template <int C>
__device__ __forceinline__ void chan_store(bf16* p, const float (&x)[C]) {
  if constexpr (C == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
  else if constexpr (C == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
  else *reinterpret_cast<uint32_t*>(p) = pack2(x[0], x[1]);
}
template <int C>
__device__ __forceinline__ float chan(const Chans<C>& x, int e) {
  return __uint_as_float(e % 2 ? x.v[e / 2] & 0xFFFF0000u : x.v[e / 2] << 16);
}
template <int C>
__device__ __forceinline__ float chan_dot(const Chans<C>& x, const Chans<C>& y) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < C; ++e) s = fmaf(chan(x, e), chan(y, e), s);
  return s;
}
// Whether every lane's sums have become no number, which further terms do not change.
template <int C>
__device__ __forceinline__ bool all_nan(const float (&x)[C]) {
  bool nan = true;
#pragma unroll
  for (int e = 0; e < C; ++e) nan &= x[e] != x[e];
  return all_sync(nan);
}
// A walk over [begin, end): kWalk rows together, whose loads and sums over the lanes then overlap; `on` is asked after each of those.
constexpr int kWalk = 8;
template <class Row, class On>
__device__ __forceinline__ bool walk(int begin, int end, Row row, On on) {
  for (int i0 = begin; i0 < end; i0 += kWalk) {
    if (i0 + kWalk <= end) {
#pragma unroll
      for (int i = 0; i < kWalk; ++i) row(i0 + i);
    } else {
      for (int i = i0; i < end; ++i) row(i);
    }
    if (!on()) return false;
  }
  return true;
}

// Unit of a persistent block's round: every other round backwards, so that no block has the longest unit of each.
__device__ __forceinline__ int unit_of(int round) {
  const int g = gridDim.x, b = blockIdx.x;
  return round * g + (round & 1 ? g - 1 - b : b);
}

// The tail of a kernel whose waits are bounded: see umma_gemm.cuh.
__device__ __forceinline__ void finish(int tid, int warp, volatile int* abort_flag, int* status, uint32_t tmem, int cols) {
  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // (copies and MMAs in flight)
    if (tid == 0) report_timeout(status);
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
// Two blocks an SM, each with one query tile of a head: one's softmax runs beside the other's products.  Warp 0 issues
// the TMA loads, warp 1 the MMAs, warps 2..5 own a row a thread.  S of the next key tile is issued behind O += P V of this
// one (P lies in S's columns: the tensor cores work in order); K and V pass through a ring.
// Measured (52 heads, 2 sequences, k = 8, 319 steps of 128 keys an SM): 450 us by itself, 500 in calls back to back, where the power
// limit takes the clock down.  By themselves too: one persistent block an SM with two query tiles that share the ring, four
// warps a tile 510, eight 541, steps of 64 keys with two buffers of scores 639 (an MMA of 64 columns takes as long as one of
// 128); a quarter of the exponentials as polynomials on the FMA units 485.
// What bounds it: of 2400 cycles a step and SM (3300 where a query tile has five steps: 13B heads, 4 sequences of 213-420
// groups) the MMAs are 1024 and the exponentials (16 a cycle) as many; the rest is the latency of the two hand-overs between
// the warps and the tensor cores, which the second block hides in part, and a query tile's beginning and end.
template <int D>
struct Fwd {
  static constexpr int NS = D == 128 ? 2 : 4;   // slots of the ring
  static constexpr int threads = 192, cols = 256;
  static constexpr int smem = (1 + NS) * kTileBytes<D> + 2048;
};
struct FwdCtl {
  uint64_t full[4], empty[4], q_full, s_full, p_full, o_full;
  uint32_t tmem;
  int abort_flag;
};

// out of row r of the query tile over its key tiles [i0, i1), by one warp and over the keys it sees alone (their lse is there).
template <int D>
__device__ __noinline__ void fwd_row(const AttnArgs& a, const TcArgs& t, const QueryWork u, int r) {
  constexpr int C = D / 32;
  const int lane = threadIdx.x & 31, h = u.h;
  const size_t row_q = (size_t)u.qrow + r, at = ((size_t)u.split * a.n_heads + h) * a.rows + row_q;
  const float lse = t.splits == 1 ? a.lse[at] : t.part_l[at];
  const TileRow tr(r, u.w.R);
  const bf16 *k = (const bf16*)a.k + (size_t)(h / a.per) * D + C * lane, *v = (const bf16*)a.v + (size_t)(h / a.per) * D + C * lane;
  const Chans<C> q = chan_load<C>((const bf16*)a.q + row_q * a.ldq + (size_t)h * D + C * lane);
  float o[C];
#pragma unroll
  for (int e = 0; e < C; ++e) o[e] = 0.f;
  bool on = lse > -INFINITY;   // (else this part of the keys has none that counts)
  for (int i = u.i0; on && i < u.i1; ++i) {
    int x0, n, lo, hi;
    const int kind = u.w.tile(i, u.group, u.rows, x0, n);
    tr.sees(kind, x0, n, u.group, u.rows, lo, hi);
    on = walk(lo, hi + 1, [&](int c) {
      const size_t row = u.w.key_row(kind, x0 + c);
      const Chans<C> x = chan_load<C>(k + row * a.ldk), y = chan_load<C>(v + row * a.ldv);
      const float p = exp2f((warp_sum(chan_dot(q, x)) * a.scale - lse) * kLog2e);
#pragma unroll
      for (int e = 0; e < C; ++e) o[e] = fmaf(p, chan(y, e), o[e]);
    }, [&] { return !all_nan(o); });
  }
  if (t.splits == 1) {
    chan_store<C>((bf16*)a.out + row_q * a.ldo + (size_t)h * D + C * lane, o);
  } else {
#pragma unroll
    for (int e = 0; e < C; ++e) t.part_o[at * D + C * lane + e] = o[e];
  }
}

template <int D>
__global__ void __launch_bounds__(Fwd<D>::threads, 2)
k_gat_fwd(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
          const __grid_constant__ TcArgs t) {
  using F = Fwd<D>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
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
  }
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, F::cols);
    fence_before_sync();
  }
  const QueryWork u(s, a, t, blockIdx.x);
  const int i0 = u.i0, i1 = u.i1, rows = u.rows, group = u.group, qrow = u.qrow;
  __syncthreads();
  fence_after_sync();
  pdl_launch_dependents();   // (with its tensor memory in hand: the next kernel's blocks take theirs before they wait for this one)
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_o = tmem + kT;
  volatile int* abort_flag = &ctl.abort_flag;
  pdl_wait();

  if (warp == 0) {
    if (lane == 0 && i0 < i1) {
      load_rows<D>(sq, &maps.q, qrow, u.h * D, &ctl.q_full);
      const int col = u.h / a.per * D;
      int it = 0;
      bool ok = true;
      for (int i = i0; ok && i < i1; ++i) {
        int x0, n;
        const int kind = u.w.tile(i, group, rows, x0, n), row0 = kind == CTX ? u.w.kv0 : u.w.g0;
        for (int kv = 0; ok && kv < 2; ++kv, ++it) {
          const int slot = it % F::NS;
          ok = mbar_wait(&ctl.empty[slot], ((it / F::NS) & 1) ^ 1, abort_flag);
          if (ok) load_keys<D>(ring + slot * kTileBytes<D>, kv ? &maps.v : &maps.k, kv ? &maps.vs : &maps.ks, kind, row0, s.R, x0, col,
                               &ctl.full[slot]);
        }
      }
    }
  } else if (warp == 1) {
    // (the whole warp walks, so that addresses and descriptors stay in uniform registers; one lane issues)
    const bool leader = elect_one();
    const int n = i1 - i0;
    const uint64_t dq = desc_k(sq), dk = desc_k(ring), dv = desc_mn(ring);
    bool ok = n > 0 && all_sync(mbar_wait(&ctl.q_full, 0, abort_flag));
    auto scores = [&](int i) {
      const int it = 2 * i, slot = it % F::NS;
      ok = all_sync(mbar_wait(&ctl.full[slot], (it / F::NS) & 1, abort_flag));
      if (!ok) return;
      fence_after_sync();
      if (leader) {
        mma_scores<D>(tmem, dq, dk + slot * (kTileBytes<D> >> 4));
        mma_commit(&ctl.s_full);
        mma_commit(&ctl.empty[slot]);
      }
      __syncwarp();
    };
    if (ok) scores(0);
    for (int i = 0; ok && i < n; ++i) {
      const int it = 2 * i + 1, slot = it % F::NS;
      ok = all_sync(mbar_wait(&ctl.full[slot], (it / F::NS) & 1, abort_flag)) && all_sync(mbar_wait(&ctl.p_full, i & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      if (leader) {
        mma_sums<D, kT>(t_o, tmem, dv + slot * (kTileBytes<D> >> 4), i > 0);
        mma_commit(&ctl.empty[slot]);
        if (i + 1 == n) mma_commit(&ctl.o_full);
      }
      __syncwarp();
      if (i + 1 < n) scores(i + 1);
    }
  } else {
    const int q = warp & 3, r = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16, ts = tmem + lanes, to = t_o + lanes;
    const float c = a.scale * kLog2e;
    const TileRow tr(r, s.R);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int i = i0; i < i1; ++i) {
      int x0, n, lo, hi;
      const int kind = u.w.tile(i, group, rows, x0, n);
      tr.sees(kind, x0, n, group, rows, lo, hi);
      const bool whole = all_sync(lo <= 0 && hi >= kT - 1);
      ok = all_sync(mbar_wait(&ctl.s_full, (i - i0) & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      uint32_t v[kT];
#pragma unroll
      for (int j = 0; j < kT; j += 32) ld32(ts + j, v + j);
      ld_wait();
      if (!whole) {
#pragma unroll
        for (int j = 0; j < kT; j += 32)
          if (chunk_sees(j, lo, hi) != kAll) mask_scores(v + j, j, lo, hi);
      }
      float y[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < kT; j += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = max3(y[e], __uint_as_float(v[j + e]), __uint_as_float(v[j + 4 + e]));
      const float top = fmaxf(max3(y[0], y[1], y[2]), y[3]);
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
          for (int j = 0; j < D; j += 16) {
            uint32_t o[16];
            ld16(to + j, o);
            ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            st16(to + j, o);
          }
        }
      }
      float ref = m > -INFINITY ? m * c : 0.f;
      // (v c - ref is what ref's rounding left where the two are equal: nothing that counts up to kFar, and beyond single
      // precision's exponents from 2^31 on)
      if (__any_sync(0xffffffffu, fabsf(ref) > kFar)) {
        const float far = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int j = 0; j < kT; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) - far);
        ref = 0.f;
      }
      f2 sum0 = {0.f, 0.f}, sum1 = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kT; j += 32) {
        uint32_t p[16];
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const f2 z0 = fma2(pair_of(v + j + e), f2{c, c}, f2{-ref, -ref}), z1 = fma2(pair_of(v + j + e + 2), f2{c, c}, f2{-ref, -ref});
          const f2 w0 = {ex2(z0.x), ex2(z0.y)}, w1 = {ex2(z1.x), ex2(z1.y)};
          sum0 = add2(sum0, w0);
          sum1 = add2(sum1, w1);
          p[e / 2] = pack2(w0.x, w0.y);
          p[e / 2 + 1] = pack2(w1.x, w1.y);
        }
        st16(ts + j / 2, p);
      }
      l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
      st_wait();
      fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full);
    }
    if (ok && i0 < i1) ok = all_sync(mbar_wait(&ctl.o_full, 0, abort_flag));
    if (ok) {
      fence_after_sync();
      // (no sum: a part of the keys of which the row sees none leaves zeros, which the join passes over; a row whose scores
      // are all -inf has no probabilities, and is no number)
      const float inv = l == 0.f ? t.none : 1.f / l;
      const size_t row = (size_t)qrow + r, at = ((size_t)u.split * a.n_heads + u.h) * a.rows + row;
      bf16* dst = (bf16*)a.out + row * a.ldo + (size_t)u.h * D;
      float odd = 0.f;                       // no number once a sum is not finite
#pragma unroll
      for (int j = 0; j < D; j += 32) {
        uint32_t o[32];
        float y[32];
        if (i0 < i1) {
          ld32(to + j, o);
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
        const float lse = l == 0.f ? -INFINITY : fmaf(m, a.scale, log2f(l) * kLn2);
        if (t.splits == 1) a.lse[(size_t)u.h * a.rows + row] = lse;
        else t.part_l[at] = lse;
      }
      // (where l is no number, or a row has none, all of it is no number, and so it came out)
      unsigned bad = __ballot_sync(0xffffffffu, r < rows && odd != 0.f && inv == inv);
      __syncwarp();
      for (; bad; bad &= bad - 1) fwd_row<D>(a, t, u, 32 * q + __ffs(bad) - 1);
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
// A persistent block an SM, one query tile of a head at a time.  Four groups of four warps share a tile's rows, a quarter of
// the keys each.  The scores pass through registers, so that the next tile's are formed as soon as they are read; dP has
// two buffers, and dS takes dP's columns (each quarter its own): the tensor cores work on S, dP of the next tile and dQ of the
// last one while the warps turn this one's into dS.
// Measured: 13B heads, 4 sequences of 213-420 groups of 5 rows, 187 us; 2047 groups on 8 key heads 315.  Steps of 64 keys in three
// buffers, two groups of warps taking turns: a fifth and two fifths more.  What bounds it: 3950 and 3100 cycles a step of which the
// MMAs are 1536 and the exponentials 1024; the rest is the latency of the loads from tensor memory, stores to it and barriers.
template <int D>
struct Dq {
  static constexpr int NK = 3, NV = 2, threads = 576;
  static constexpr int smem = (2 + NK + NV) * kTileBytes<D> + 2048;
};
struct DqCtl {
  uint64_t k_full[3], k_empty[3], v_full[2], v_empty[2], q_full, q_empty, s_empty, dp_full[2], ds_full, o_full, o_empty;   // (dp_full: S and dP)
  uint32_t tmem;
  int abort_flag;
};

template <int D>
__global__ void __launch_bounds__(Dq<D>::threads, 1)
k_gat_dq(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
         const __grid_constant__ TcArgs t) {
  using F = Dq<D>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t sq = base, so = sq + kTileBytes<D>, sk = so + kTileBytes<D>, sv = sk + F::NK * kTileBytes<D>;
  DqCtl& ctl = *reinterpret_cast<DqCtl*>(smem_raw + (base - raw) + (2 + F::NK + F::NV) * kTileBytes<D>);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < F::NK; ++i) { mbar_init(&ctl.k_full[i], 1); mbar_init(&ctl.k_empty[i], 1); }
    for (int i = 0; i < F::NV; ++i) { mbar_init(&ctl.v_full[i], 1); mbar_init(&ctl.v_empty[i], 1); }
    mbar_init(&ctl.q_full, 2);
    mbar_init(&ctl.q_empty, 1);
    mbar_init(&ctl.s_empty, 16);
    mbar_init(&ctl.dp_full[0], 1);
    mbar_init(&ctl.dp_full[1], 1);
    mbar_init(&ctl.ds_full, 16);
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.o_empty, 16);
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, 512);
    fence_before_sync();
  }
  __syncthreads();
  fence_after_sync();
  pdl_launch_dependents();   // (with its tensor memory in hand: the next kernel's blocks take theirs before they wait for this one)
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_dp = tmem + kT, t_o = tmem + 3 * kT;
  volatile int* abort_flag = &ctl.abort_flag;
  const int units = QueryWork::count(s, a, t);
  pdl_wait();

  if (warp == 0) {
    if (lane == 0) {
      int it = 0, nu = 0;
      bool ok = true;
      for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
        if (unit >= units) continue;
        const QueryWork u(s, a, t, unit);
        if (u.i0 == u.i1) continue;
        ok = mbar_wait(&ctl.q_empty, (nu++ & 1) ^ 1, abort_flag);
        if (!ok) break;
        load_rows<D>(sq, &maps.q, u.qrow, u.h * D, &ctl.q_full);
        load_rows<D>(so, &maps.dout, u.qrow, u.h * D, &ctl.q_full);
        const int col = u.h / a.per * D;
        for (int i = u.i0; i < u.i1; ++i, ++it) {
          int x0, n;
          const int kind = u.w.tile(i, u.group, u.rows, x0, n), row0 = kind == CTX ? u.w.kv0 : u.w.g0, ks = it % F::NK, vs = it % F::NV;
          ok = mbar_wait(&ctl.k_empty[ks], ((it / F::NK) & 1) ^ 1, abort_flag);
          if (!ok) break;
          load_keys<D>(sk + ks * kTileBytes<D>, &maps.k, &maps.ks, kind, row0, s.R, x0, col, &ctl.k_full[ks]);
          ok = mbar_wait(&ctl.v_empty[vs], ((it / F::NV) & 1) ^ 1, abort_flag);
          if (!ok) break;
          load_keys<D>(sv + vs * kTileBytes<D>, &maps.v, &maps.vs, kind, row0, s.R, x0, col, &ctl.v_full[vs]);
        }
      }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();   // (see the forward kernel)
    int it = 0, nu = 0;   // tiles and units so far
    bool ok = true;
    const uint64_t dq = desc_k(sq), dg = desc_k(so), dk = desc_k(sk), dv = desc_k(sv), dkm = desc_mn(sk);
    constexpr int kStep = kTileBytes<D> >> 4;
    // S and dP of tile number i (over all units)
    auto issue = [&](int i, bool last) {
      const int ks = i % F::NK, vs = i % F::NV;
      ok = all_sync(mbar_wait(&ctl.s_empty, (i & 1) ^ 1, abort_flag)) && all_sync(mbar_wait(&ctl.k_full[ks], (i / F::NK) & 1, abort_flag));
      if (!ok) return;
      fence_after_sync();
      if (leader) mma_scores<D>(tmem, dq, dk + ks * kStep);
      __syncwarp();
      ok = all_sync(mbar_wait(&ctl.v_full[vs], (i / F::NV) & 1, abort_flag));
      if (!ok) return;
      fence_after_sync();
      if (leader) {
        mma_scores<D>(t_dp + (i & 1) * kT, dg, dv + vs * kStep);
        mma_commit(&ctl.dp_full[i & 1]);
        mma_commit(&ctl.v_empty[vs]);
        if (last) mma_commit(&ctl.q_empty);
      }
      __syncwarp();
    };
    for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
      if (unit >= units) continue;
      const QueryWork u(s, a, t, unit);
      const int cnt = u.i1 - u.i0;
      if (cnt == 0) continue;
      ok = all_sync(mbar_wait(&ctl.q_full, nu & 1, abort_flag));
      if (ok) issue(it, cnt == 1);
      for (int i = 0; ok && i < cnt; ++i, ++it) {
        if (i + 1 < cnt) issue(it + 1, i + 2 == cnt);
        ok = ok && all_sync(mbar_wait(&ctl.ds_full, it & 1, abort_flag));
        if (ok && i == 0) ok = all_sync(mbar_wait(&ctl.o_empty, (nu & 1) ^ 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        const int ks = it % F::NK;
        if (leader) {
          mma_sums<D, 32>(t_o, t_dp + (it & 1) * kT, dkm + ks * kStep, i > 0);
          mma_commit(&ctl.k_empty[ks]);
          if (i + 1 == cnt) mma_commit(&ctl.o_full);
        }
        __syncwarp();
      }
      ++nu;
    }
  } else {
    const int q = warp & 3, quarter = (warp - 2) >> 2, r = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16, mine = lanes + 32 * quarter;
    const float c = a.scale * kLog2e;
    const TileRow tr(r, s.R);
    int it = 0, nu = 0;
    bool ok = true;
    for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
      if (unit >= units) continue;
      const QueryWork u(s, a, t, unit);
      const int rows = u.rows, cnt = u.i1 - u.i0;
      const size_t row = (size_t)u.qrow + r, at = (size_t)u.h * a.rows + row;
      const float lse = r < rows ? a.lse[at] * kLog2e : 0.f, delta = r < rows ? a.delta[at] : 0.f;
      for (int i = u.i0; i < u.i1; ++i, ++it) {
        const uint32_t td = t_dp + (it & 1) * kT + mine;
        ok = all_sync(mbar_wait(&ctl.dp_full[it & 1], (it >> 1) & 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        uint32_t v[32], d[32], p[16];
        ld32(tmem + mine, v);
        ld32(td, d);
        int x0, n, lo, hi;
        const int kind = u.w.tile(i, u.group, rows, x0, n);
        tr.sees(kind, x0, n, u.group, rows, lo, hi);
        lo -= 32 * quarter;
        hi -= 32 * quarter;
        const bool whole = all_sync(lo <= 0 && hi >= 31);
        ld_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.s_empty);
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          const f2 z = fma2(pair_of(v + j), f2{c, c}, f2{-lse, -lse});
          v[j] = __float_as_uint(ex2(z.x));
          v[j + 1] = __float_as_uint(ex2(z.y));
        }
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const f2 z = mul2(pair_of(v + e), add2(pair_of(d + e), f2{-delta, -delta}));
          d[e] = __float_as_uint(z.x);
          d[e + 1] = __float_as_uint(z.y);
        }
        if (!whole) mask_zero(d, 0, lo, hi);
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = pack2(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
        st16(td, p);
        st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.ds_full);
      }
      if (ok && cnt > 0) ok = all_sync(mbar_wait(&ctl.o_full, nu++ & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      constexpr int N = D / 4;
      float* part = t.part_o + (((size_t)u.split * a.n_heads + u.h) * a.rows + row) * D + N * quarter;
      bf16* dst = (bf16*)a.dq + row * a.lddq + (size_t)u.h * D + N * quarter;
      float odd = 0.f, y[N];
      uint32_t o[N];
      if (cnt > 0) {
        ldn<N>(t_o + lanes + N * quarter, o);
        ld_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.o_empty);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = 0;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        odd = fmaf(__uint_as_float(o[e]), 0.f, odd);
        y[e] = __uint_as_float(o[e]) * a.scale;
      }
      if (r < rows) {
        if (t.splits == 1) {
          store_bf16<N>(dst, y);
        } else {
#pragma unroll
          for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(part + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
        }
      }
      // (where lse or delta is no number, the whole row is, and so it came out)
      const unsigned bad = __ballot_sync(0xffffffffu, r < rows && odd != 0.f && lse == lse && delta == delta);
      if (lane == 0) {
        const int at_unit = units - 1 - unit, lot = 4 * (at_unit / t.splits) + q;
        t.bad[4 * ((size_t)lot * t.splits + at_unit % t.splits) + quarter] = bad;
        if (bad) {
          t.where[lot] = Where{u.qrow + 32 * q, 1, u.h};
          *a.any = 1;
        }
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

// ---- backward: dk, dv of the masks, delta ------------------------------------------------------------------
// A [MASK] row is seen by the R - j rows of its own group that follow it: too little for a matrix product.  A warp per
// (group, key head) keeps the group's keys, values and their gradients in registers, a lane D / 32 neighbouring
// channels; it also forms delta = dout . out of the rows it reads anyway.
// Measured: 6650 rows of 40 heads 121 us (409 MB, 3.4 TB/s); 10235 rows of 32 heads on 8, 98 us.  Bound by the latency of a
// warp's loads: its registers leave room for 12 warps an SM (with spills at 16 and 20 it took 129 and 136 us).
// delta of the rows with few keys (see kExactKeys): the first groups of sequences with a short context.  A warp per (row, head).
__host__ __device__ inline int few_groups(int ctx, int groups) { return ctx >= kExactKeys ? 0 : (groups < kExactKeys - ctx ? groups : kExactKeys - ctx); }
template <int D>
__global__ void __launch_bounds__(256) k_gat_few(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int u = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (u >= s.tile0[s.B] * a.n_heads) return;            // tile0: such rows before the sequence
  const int i = u / a.n_heads, h = u - i * a.n_heads, b = seq_of_tile(s, i), rho = i - s.tile0[b];
  const int n = s.ctx[b] + rho / s.R + 1 + rho % s.R;
  if (n > kExactKeys) return;
  const float d = delta_of_keys<bf16, D>(s, a, b, rho, h, n);
  if (lane == 0) a.delta[(size_t)h * a.rows + s.q0[b] + rho] = d;
}

// Sums of N values (a power of two) over the warp: lane l ends with the sum of value l % N.  At each step a lane passes on the
// half of its values that the other one keeps: N + 4 exchanges at most where one value at a time takes 5 N.
template <int N>
__device__ __forceinline__ float sum_many(float (&v)[N], int lane) {
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1) {
    const bool up = lane & n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, n);
    }
  }
  float s = v[0];
#pragma unroll
  for (int o = N; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

// A warp per (group, key head), C channels a lane; RM: most rows of a group that the registers hold.  A row's scores and
// dP of all masks it sees, and its delta, are summed over the lanes together; lane j - 1 then has mask j's.
template <int D, int RM>
__global__ void __launch_bounds__(128, RM <= 3 ? 4 : (RM <= 5 ? 3 : 2))
k_gat_masks(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a, int groups) {
  constexpr int C = D / 32, NM = RM - 1;                          // NM: masks
  constexpr int N = NM <= 1 ? 4 : (NM <= 3 ? 8 : (NM <= 7 ? 16 : 32));   // scores, dP, delta
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x % 32, R = s.R;
  const long long unit = (long long)blockIdx.x * 4 + threadIdx.x / 32;
  if (unit == 0 && lane == 0) *a.any = 0;   // (for the kernels behind this one)
  if (unit >= (long long)groups * a.n_kv) return;
  const int g = (int)(unit / a.n_kv), hk = (int)(unit - (long long)g * a.n_kv);
  int lo = 0, hi = s.B - 1;            // the sequence of group g: its rows begin at q0 / R
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.q0[mid] <= g * R) lo = mid; else hi = mid - 1;
  }
  const size_t q0 = (size_t)g * R, k0 = (size_t)s.kv0[lo] + s.ctx[lo] + (q0 - s.q0[lo]);
  const int n0 = s.ctx[lo] + g - s.q0[lo] / R + 1;   // keys that the group's first row sees
  Chans<C> k[RM], v[RM];
  float dk[RM][C], dv[RM][C];
#pragma unroll
  for (int j = 1; j < RM; ++j) {
    if (j < R) {
      k[j] = chan_load<C>((const bf16*)a.k + (k0 + j) * a.ldk + (size_t)hk * D + C * lane);
      v[j] = chan_load<C>((const bf16*)a.v + (k0 + j) * a.ldv + (size_t)hk * D + C * lane);
    }
#pragma unroll
    for (int e = 0; e < C; ++e) dk[j][e] = dv[j][e] = 0.f;
  }
  const float c = a.scale * kLog2e;
  for (int h = hk * a.per; h < (hk + 1) * a.per; ++h) {
    float* delta_out = a.delta + (size_t)h * a.rows + q0;
    const float lse = lane < R ? a.lse[(size_t)h * a.rows + q0 + lane] * kLog2e : 0.f;   // lane i: of row i
    const bf16 *q_in = (const bf16*)a.q + q0 * a.ldq + (size_t)h * D + C * lane,
               *g_in = (const bf16*)a.dout + q0 * a.lddo + (size_t)h * D + C * lane,
               *o_in = (const bf16*)a.out + q0 * a.ldo + (size_t)h * D + C * lane;
    constexpr int NB = RM <= 5 ? RM : 4;       // rows whose values are in flight
#pragma unroll
    for (int i0 = 0; i0 < RM; i0 += NB) {
      if (i0 >= R) break;
      Chans<C> q[NB], d[NB], o[NB];
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const int i = i0 + x;
        if (i < RM && i < R) {
          d[x] = chan_load<C>(g_in + i * a.lddo);
          o[x] = chan_load<C>(o_in + i * a.ldo);
          if (i > 0) q[x] = chan_load<C>(q_in + i * a.ldq);
        }
      }
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const int i = i0 + x;
        if (i >= RM || i >= R) break;
        if (i == 0) {
          float delta = chan_dot(d[x], o[x]);
#pragma unroll
          for (int w = 16; w > 0; w >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, w);
          if (lane == 0 && n0 > kExactKeys) delta_out[0] = delta;
          continue;
        }
        float t[N];
#pragma unroll
        for (int y = 0; y < N; ++y) t[y] = 0.f;
#pragma unroll
        for (int j = 1; j < RM; ++j) {
          if (j > i) break;
          t[j - 1] = chan_dot(q[x], k[j]);
          t[NM + j - 1] = chan_dot(d[x], v[j]);
        }
        t[2 * NM] = chan_dot(d[x], o[x]);
        const float sum = sum_many<N>(t, lane);
        float delta = __shfl_sync(0xffffffffu, sum, 2 * NM);
        const bool few = n0 + i <= kExactKeys;        // (k_gat_few has it)
        if (few) delta = delta_out[i];
        const float dp = __shfl_sync(0xffffffffu, sum, (lane + NM) & (N - 1)),
                    ls = __shfl_sync(0xffffffffu, lse, i);
        if (lane == 0 && !few) delta_out[i] = delta;
        const float p = ex2(fmaf(sum, c, -ls)), ds = p * (dp - delta);    // lane j - 1: of mask j
#pragma unroll
        for (int j = 1; j < RM; ++j) {
          if (j > i) break;
          const float pj = __shfl_sync(0xffffffffu, p, j - 1), dsj = __shfl_sync(0xffffffffu, ds, j - 1);
#pragma unroll
          for (int e = 0; e < C; ++e) {
            dv[j][e] = fmaf(pj, chan(d[x], e), dv[j][e]);
            dk[j][e] = fmaf(dsj, chan(q[x], e), dk[j][e]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int j = 1; j < RM; ++j) {
    if (j >= R) break;
#pragma unroll
    for (int e = 0; e < C; ++e) dk[j][e] *= a.scale;
    chan_store<C>((bf16*)a.dk + (k0 + j) * a.lddk + (size_t)hk * D + C * lane, dk[j]);
    chan_store<C>((bf16*)a.dv + (k0 + j) * a.lddv + (size_t)hk * D + C * lane, dv[j]);
  }
}

// ---- backward: dk, dv -----------------------------------------------------------------------------------
// A persistent block an SM, one key tile (context or real rows) and key head at a time, or a part of its steps:
// the query tiles of all heads that share the key head.  Tensor memory is full with S^T (P^T in its columns), dP^T (dS^T
// in its columns), dK and dV.  The warps form P^T while the tensor cores work on dK and dP^T, and dS^T while they work on
// dV and the next step's S^T.  A thread owns a key and a quarter of the query columns, whose lse and delta a
// warp of its own puts into shared memory.
// Measured: 13B heads, 4 sequences of 213-420 groups of 5 rows, 187 us; 2047 groups on 8 key heads 329, in one part per key tile
// 576 (the first tiles are seen by all 10235 rows of four heads, the last ones by few).  Steps of 64 rows with two groups of
// warps taking turns: a fifth and a quarter more.  What bounds it: 5000 and 3650 cycles a step, of which the MMAs are 2048; tensor memory has no room
// for a second step's scores of 128 rows, so that the two halves of a step wait for each other's products.
template <int D>
struct Dkv {
  static constexpr int threads = 608;
  static constexpr int smem = 6 * kTileBytes<D> + 1024 + 2 * 2 * kT * 4 + 1024;
};
struct DkvCtl {
  uint64_t q_full[2], q_empty[2], g_full[2], g_empty[2], t_full[2], t_empty[2], k_full, k_empty, s_full, p_full, dp_full, ds_full,
      o_full, o_empty;
  uint32_t tmem;
  int abort_flag;
};

struct KeyWork {
  int b, hk, part, parts, slot;        // slot: of its sums, if there is more than one part
  int kind, x0, n, row0, step, q_begin, q_end, per_head, j0, j1;
  __device__ static int count(const Seqs& s, const AttnArgs& a, const TcArgs& t) { return s.tile0[s.B] * a.n_kv * t.parts; }
  __device__ KeyWork(const Seqs& s, const AttnArgs& a, const TcArgs& t, int unit) {
    // (the first tiles of a sequence are seen by the most rows: parts of all heads side by side, tiles in order)
    const int tile = unit / (a.n_kv * t.parts), i = unit - tile * a.n_kv * t.parts;
    hk = i / t.parts;
    part = i - hk * t.parts;
    slot = unit;
    b = seq_of_tile(s, tile);
    const int ctx = s.ctx[b], groups = s.groups[b], R = s.R, x = tile - s.tile0[b], n_ctx = div_up(ctx, kT);
    step = 1;
    q_begin = 0;
    q_end = groups * R;
    if (x < n_ctx) { kind = CTX; x0 = x * kT; n = min(kT, ctx - x0); row0 = s.kv0[b] + x0; }
    else { kind = REAL; x0 = (x - n_ctx) * kT; n = min(kT, groups - x0); step = R; row0 = s.kv0[b] + ctx + x0 * R; q_begin = x0 * R; }
    per_head = div_up(q_end - q_begin, kT);
    const int cnt = per_head * a.per;
    parts = max(1, div_up(cnt, t.cap));
    j0 = min(cnt, part * t.cap);
    j1 = min(cnt, j0 + t.cap);
    if (t.parts == 1) { parts = 1; j0 = 0; j1 = cnt; }
  }
  __device__ bool there() const { return part < parts; }
  // Walks the steps: head and first query row (of the sequence).
  struct Step {
    int h, r0, q_begin, q_end;
    __device__ Step(const KeyWork& u, int per) {
      const int hh = u.j0 / max(1, u.per_head);
      h = u.hk * per + hh;
      q_begin = u.q_begin;
      q_end = u.q_end;
      r0 = q_begin + (u.j0 - hh * u.per_head) * kT;
    }
    __device__ void next() {
      r0 += kT;
      if (r0 >= q_end) { r0 = q_begin; ++h; }
    }
  };
  // Query rows that see key i of the tile: [lo, hi].
  __device__ void seen(int i, int R, int& lo, int& hi) const {
    lo = kind == REAL ? (x0 + i) * R : 0;
    hi = i < n ? q_end - 1 : -1;
  }
};

template <int D>
__global__ void __launch_bounds__(Dkv<D>::threads, 1)
k_gat_dkv(const __grid_constant__ Maps maps, const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
          const __grid_constant__ TcArgs t) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t sk = base, sv = sk + kTileBytes<D>, sq = sv + kTileBytes<D>, sg = sq + 2 * kTileBytes<D>;
  float* s_stat = reinterpret_cast<float*>(smem_raw + (base - raw) + 6 * kTileBytes<D>);   // [slot][-lse, -delta][128]
  DkvCtl& ctl = *reinterpret_cast<DkvCtl*>(s_stat + 2 * 2 * kT);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.q_full[i], 1); mbar_init(&ctl.q_empty[i], 1);
      mbar_init(&ctl.g_full[i], 1); mbar_init(&ctl.g_empty[i], 1);
      mbar_init(&ctl.t_full[i], 32); mbar_init(&ctl.t_empty[i], 16);
    }
    mbar_init(&ctl.k_full, 2);
    mbar_init(&ctl.k_empty, 1);
    mbar_init(&ctl.s_full, 1);
    mbar_init(&ctl.p_full, 16);
    mbar_init(&ctl.dp_full, 1);
    mbar_init(&ctl.ds_full, 16);
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.o_empty, 16);
    ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    __syncwarp();
    alloc_tmem(&ctl.tmem, 512);
    fence_before_sync();
  }
  __syncthreads();
  fence_after_sync();
  pdl_launch_dependents();   // (with its tensor memory in hand: the next kernel's blocks take theirs before they wait for this one)
  const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, t_dp = tmem + kT, t_dk = tmem + 2 * kT, t_dv = tmem + 3 * kT;
  volatile int* abort_flag = &ctl.abort_flag;
  const int units = KeyWork::count(s, a, t);
  pdl_wait();

  if (warp == 0) {
    if (lane == 0) {
      int it = 0, nu = 0;
      bool ok = true;
      for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
        if (unit >= units) continue;
        const KeyWork u(s, a, t, unit);
        if (!u.there() || u.j0 == u.j1) continue;
        ok = mbar_wait(&ctl.k_empty, (nu++ & 1) ^ 1, abort_flag);
        if (!ok) break;
        const int base_row = u.kind == CTX ? s.kv0[u.b] : s.kv0[u.b] + s.ctx[u.b];
        load_keys<D>(sk, &maps.k, &maps.ks, u.kind, base_row, s.R, u.x0, u.hk * D, &ctl.k_full);
        load_keys<D>(sv, &maps.v, &maps.vs, u.kind, base_row, s.R, u.x0, u.hk * D, &ctl.k_full);
        KeyWork::Step x(u, a.per);
        for (int j = u.j0; j < u.j1; ++j, ++it, x.next()) {
          const int r0 = s.q0[u.b] + x.r0, col = x.h * D, slot = it & 1;
          const uint32_t parity = ((it >> 1) & 1) ^ 1;
          ok = mbar_wait(&ctl.q_empty[slot], parity, abort_flag);
          if (!ok) break;
          load_rows<D>(sq + slot * kTileBytes<D>, &maps.q, r0, col, &ctl.q_full[slot]);
          ok = mbar_wait(&ctl.g_empty[slot], parity, abort_flag);
          if (!ok) break;
          load_rows<D>(sg + slot * kTileBytes<D>, &maps.dout, r0, col, &ctl.g_full[slot]);
        }
      }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    int it = 0, nu = 0;
    bool ok = true;
    const uint64_t dk = desc_k(sk), dv = desc_k(sv), dq = desc_k(sq), dg = desc_k(sg), dqm = desc_mn(sq), dgm = desc_mn(sg);
    constexpr int kStep = kTileBytes<D> >> 4;
    auto scores = [&](int i) {
      ok = ok && all_sync(mbar_wait(&ctl.q_full[i & 1], (i >> 1) & 1, abort_flag));
      if (!ok) return;
      fence_after_sync();
      if (leader) {
        mma_scores<D>(tmem, dk, dq + (i & 1) * kStep);
        mma_commit(&ctl.s_full);
      }
      __syncwarp();
    };
    auto dprob = [&](int i, bool last) {
      ok = ok && all_sync(mbar_wait(&ctl.g_full[i & 1], (i >> 1) & 1, abort_flag));
      if (!ok) return;
      fence_after_sync();
      if (leader) {
        mma_scores<D>(t_dp, dv, dg + (i & 1) * kStep);
        mma_commit(&ctl.dp_full);
        if (last) mma_commit(&ctl.k_empty);
      }
      __syncwarp();
    };
    for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
      if (unit >= units) continue;
      const KeyWork u(s, a, t, unit);
      const int cnt = u.j1 - u.j0;
      if (!u.there() || cnt == 0) continue;
      ok = all_sync(mbar_wait(&ctl.k_full, nu & 1, abort_flag));
      scores(it);
      dprob(it, cnt == 1);
      for (int i = 0; ok && i < cnt; ++i, ++it) {
        ok = all_sync(mbar_wait(&ctl.p_full, it & 1, abort_flag));
        if (ok && i == 0) ok = all_sync(mbar_wait(&ctl.o_empty, (nu & 1) ^ 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        if (leader) {
          mma_sums<D, 32>(t_dv, tmem, dgm + (it & 1) * kStep, i > 0);
          mma_commit(&ctl.g_empty[it & 1]);
        }
        __syncwarp();
        if (i + 1 < cnt) scores(it + 1);
        ok = ok && all_sync(mbar_wait(&ctl.ds_full, it & 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        if (leader) {
          mma_sums<D, 32>(t_dk, t_dp, dqm + (it & 1) * kStep, i > 0);
          mma_commit(&ctl.q_empty[it & 1]);
          if (i + 1 == cnt) mma_commit(&ctl.o_full);
        }
        __syncwarp();
        if (i + 1 < cnt) dprob(it + 1, i + 2 == cnt);
      }
      ++nu;
    }
  } else if (warp == 2) {
    int it = 0;
    bool ok = true;
    for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
      if (unit >= units) continue;
      const KeyWork u(s, a, t, unit);
      if (!u.there()) continue;
      KeyWork::Step x(u, a.per);
      for (int j = u.j0; j < u.j1; ++j, ++it, x.next()) {
        const int r0 = x.r0, slot = it & 1;
        ok = all_sync(mbar_wait(&ctl.t_empty[slot], ((it >> 1) & 1) ^ 1, abort_flag));
        if (!ok) break;
        const size_t at = (size_t)x.h * a.rows + s.q0[u.b] + r0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = lane + 32 * e;
          const bool in = r0 + col < u.q_end;
          s_stat[(2 * slot) * kT + col] = in ? a.lse[at + col] * -kLog2e : 0.f;
          s_stat[(2 * slot + 1) * kT + col] = in ? -a.delta[at + col] : 0.f;
        }
        mbar_arrive(&ctl.t_full[slot]);
      }
    }
  } else {
    const int q = warp & 3, quarter = (warp - 3) >> 2, key = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16, mine = lanes + 32 * quarter;
    const float c = a.scale * kLog2e;
    int it = 0, nu = 0;
    bool ok = true;
    for (int round = 0, unit; ok && (unit = unit_of(round), round * (int)gridDim.x < units); ++round) {
      if (unit >= units) continue;
      const KeyWork u(s, a, t, unit);
      const int lot = 4 * (unit / t.parts) + q;
      uint32_t* bad_out = t.bad + 8 * ((size_t)lot * t.parts + unit % t.parts) + 2 * quarter;
      if (!u.there()) {
        if (lane == 0) bad_out[0] = bad_out[1] = 0;
        continue;
      }
      const int cnt = u.j1 - u.j0;
      int see0, see1;
      u.seen(key, s.R, see0, see1);
      KeyWork::Step x(u, a.per);
      for (int j = u.j0; j < u.j1; ++j, ++it, x.next()) {
        const int r0 = x.r0 + 32 * quarter, slot = it & 1, lo = see0 - r0, hi = see1 - r0;
        const bool whole = all_sync(lo <= 0 && hi >= 31);
        const float4 *lse = reinterpret_cast<const float4*>(s_stat + (2 * slot) * kT + 32 * quarter),
                     *delta = reinterpret_cast<const float4*>(s_stat + (2 * slot + 1) * kT + 32 * quarter);
        ok = all_sync(mbar_wait(&ctl.t_full[slot], (it >> 1) & 1, abort_flag)) && all_sync(mbar_wait(&ctl.s_full, it & 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        uint32_t v[32], d[32], p[16];
        ld32(tmem + mine, v);
        ld_wait();
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 y = lse[i / 4];
          const f2 z0 = fma2(pair_of(v + i), f2{c, c}, f2{y.x, y.y}), z1 = fma2(pair_of(v + i + 2), f2{c, c}, f2{y.z, y.w});
          v[i] = __float_as_uint(ex2(z0.x));
          v[i + 1] = __float_as_uint(ex2(z0.y));
          v[i + 2] = __float_as_uint(ex2(z1.x));
          v[i + 3] = __float_as_uint(ex2(z1.y));
        }
        if (!whole) mask_zero(v, 0, lo, hi);
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = pack2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
        st16(tmem + mine, p);
        st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.p_full);
        ok = all_sync(mbar_wait(&ctl.dp_full, it & 1, abort_flag));
        if (!ok) break;
        fence_after_sync();
        ld32(t_dp + mine, d);
        ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 y = delta[e / 4];
          const f2 z0 = mul2(pair_of(v + e), add2(pair_of(d + e), f2{y.x, y.y})),
                   z1 = mul2(pair_of(v + e + 2), add2(pair_of(d + e + 2), f2{y.z, y.w}));
          d[e] = __float_as_uint(z0.x);
          d[e + 1] = __float_as_uint(z0.y);
          d[e + 2] = __float_as_uint(z1.x);
          d[e + 3] = __float_as_uint(z1.y);
        }
        if (!whole) mask_zero(d, 0, lo, hi);
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = pack2(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
        st16(t_dp + mine, p);
        st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.ds_full);
          mbar_arrive(&ctl.t_empty[slot]);
        }
      }
      if (ok && cnt > 0) ok = all_sync(mbar_wait(&ctl.o_full, nu++ & 1, abort_flag));
      if (!ok) break;
      fence_after_sync();
      constexpr int N = D / 4;
      const bool in = key < u.n;
      const size_t row = (size_t)u.row0 + (size_t)key * u.step;
      float* part = t.part_o + ((size_t)u.slot * 2 * kT + key) * D + N * quarter;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        uint32_t x[N];
        float y[N], odd = 0.f;
        if (cnt > 0) {
          ldn<N>((kv ? t_dv : t_dk) + lanes + N * quarter, x);
          ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = 0;
        }
        if (kv && cnt > 0) {
          fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.o_empty);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
          odd = fmaf(__uint_as_float(x[e]), 0.f, odd);
          y[e] = __uint_as_float(x[e]) * (kv ? 1.f : a.scale);
        }
        if (in) {
          if (u.parts == 1) {
            store_bf16<N>((kv ? (bf16*)a.dv + row * a.lddv : (bf16*)a.dk + row * a.lddk) + (size_t)u.hk * D + N * quarter, y);
          } else {
#pragma unroll
            for (int e = 0; e < N; e += 4)
              *reinterpret_cast<float4*>(part + kv * kT * D + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
        const unsigned bad = __ballot_sync(0xffffffffu, in && odd != 0.f);
        if (lane == 0) {
          bad_out[kv] = bad;
          if (bad) {
            t.where[lot] = Where{u.row0 + 32 * q * u.step, u.step, u.hk};
            *a.any = 1;
          }
        }
      }
    }
    fence_before_sync();
  }
  finish(tid, warp, abort_flag, a.status, tmem, 512);
}

// Adds the parts of the key tiles that have several: a block per (tile, key head, 16 rows), a warp per row at a time.
template <int D>
__global__ void __launch_bounds__(256) k_gat_dkv_join(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
                                                      const __grid_constant__ TcArgs t) {
  pdl_launch_dependents();
  pdl_wait();
  const KeyWork u(s, a, t, blockIdx.x * t.parts);
  if (u.parts < 2) return;
  const int lane = threadIdx.x & 31;
  for (int i = 16 * blockIdx.y + (threadIdx.x >> 5); i < min(u.n, 16 * (int)blockIdx.y + 16); i += 8) {
    const float* part = t.part_o + ((size_t)u.slot * 2 * kT + i) * D + (D / 32) * lane;
    const size_t row = (size_t)u.row0 + (size_t)i * u.step;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float x[D / 32];
#pragma unroll
      for (int e = 0; e < D / 32; ++e) x[e] = 0.f;
      for (int p = 0; p < u.parts; ++p)
#pragma unroll
        for (int e = 0; e < D / 32; ++e) x[e] += part[((size_t)p * 2 + kv) * kT * D + e];
      chan_store<D / 32>((kv ? (bf16*)a.dv + row * a.lddv : (bf16*)a.dk + row * a.lddk) + (size_t)u.hk * D + (D / 32) * lane, x);
    }
  }
}

// ---- backward: sums that are not finite --------------------------------------------------------------------
// dq of the rows, dk and dv of the keys that k_gat_dq and k_gat_dkv left a bit for, over what the row sees (what sees the key)
// alone, by a warp each.  Sums that have become no number in every column end the walk, so that a step that is NaN throughout costs
// little more than another.  What costs is a value that reaches rows or keys by its place in a tile alone, or a part of
// the columns.  Measured (2047 groups of 5 rows, 32 heads on 8; forward and backward 0.24 + 0.77 ms): all of dout, q or k NaN
// 0.24 + 0.87, all of v 1.1 + 0.87; one NaN early in dout or q 0.24 + 17 (119 keys a head over all 40940 rows), in v 22 +
// 0.85 (all rows over all keys), in k 0.24 + 0.84.  Without one this launch takes 5 us by itself, 2 to 3 in a call.
template <int D>
__device__ __noinline__ void row_again(const Seqs& s, const AttnArgs& a, int qr, int h) {
  constexpr int C = D / 32;
  int lo = 0, hi = s.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.q0[mid] <= qr) lo = mid; else hi = mid - 1;
  }
  const int lane = threadIdx.x & 31, R = s.R, ctx = s.ctx[lo], rho = qr - s.q0[lo], t = rho / R, n = ctx + t + 1 + rho % R;
  const size_t kv0 = s.kv0[lo], g0 = kv0 + ctx;
  const bf16 *k = (const bf16*)a.k + (size_t)(h / a.per) * D + C * lane, *v = (const bf16*)a.v + (size_t)(h / a.per) * D + C * lane;
  const Chans<C> q = chan_load<C>((const bf16*)a.q + (size_t)qr * a.ldq + (size_t)h * D + C * lane),
                 g = chan_load<C>((const bf16*)a.dout + (size_t)qr * a.lddo + (size_t)h * D + C * lane);
  const float lse = a.lse[(size_t)h * a.rows + qr], delta = a.delta[(size_t)h * a.rows + qr];
  float o[C];
#pragma unroll
  for (int e = 0; e < C; ++e) o[e] = 0.f;
  walk(0, n, [&](int c) {
    const size_t row = c < ctx ? kv0 + c : (c <= ctx + t ? g0 + (size_t)(c - ctx) * R : g0 + (size_t)t * R + (c - ctx - t));
    const Chans<C> x = chan_load<C>(k + row * a.ldk), y = chan_load<C>(v + row * a.ldv);
    const float p = exp2f((warp_sum(chan_dot(q, x)) * a.scale - lse) * kLog2e), ds = p * (warp_sum(chan_dot(g, y)) - delta);
#pragma unroll
    for (int e = 0; e < C; ++e) o[e] = fmaf(ds, chan(x, e), o[e]);
  }, [&] { return !all_nan(o); });
#pragma unroll
  for (int e = 0; e < C; ++e) o[e] *= a.scale;
  chan_store<C>((bf16*)a.dq + (size_t)qr * a.lddq + (size_t)h * D + C * lane, o);
}
template <int D>
__device__ __noinline__ void key_again(const Seqs& s, const AttnArgs& a, int kr, int hk, bool want_k, bool want_v) {
  constexpr int C = D / 32;
  int lo = 0, hi = s.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.kv0[mid] <= kr) lo = mid; else hi = mid - 1;
  }
  const int lane = threadIdx.x & 31, R = s.R, ctx = s.ctx[lo], x = kr - s.kv0[lo];
  const int r_begin = x < ctx ? 0 : (x - ctx) / R * R, r_end = s.groups[lo] * R;
  const Chans<C> k = chan_load<C>((const bf16*)a.k + (size_t)kr * a.ldk + (size_t)hk * D + C * lane),
                 v = chan_load<C>((const bf16*)a.v + (size_t)kr * a.ldv + (size_t)hk * D + C * lane);
  float dk[C], dv[C];
#pragma unroll
  for (int e = 0; e < C; ++e) dk[e] = dv[e] = 0.f;
  bool on = true;
  for (int h = hk * a.per; on && h < (hk + 1) * a.per; ++h) {
    const bf16 *q_in = (const bf16*)a.q + (size_t)h * D + C * lane, *g_in = (const bf16*)a.dout + (size_t)h * D + C * lane;
    const float *lse = a.lse + (size_t)h * a.rows, *delta = a.delta + (size_t)h * a.rows;
    on = walk(r_begin, r_end, [&](int r) {
      const size_t qr = (size_t)s.q0[lo] + r;
      const Chans<C> q = chan_load<C>(q_in + qr * a.ldq), g = chan_load<C>(g_in + qr * a.lddo);
      const float p = exp2f((warp_sum(chan_dot(q, k)) * a.scale - lse[qr]) * kLog2e), ds = p * (warp_sum(chan_dot(g, v)) - delta[qr]);
#pragma unroll
      for (int e = 0; e < C; ++e) {
        dv[e] = fmaf(p, chan(g, e), dv[e]);
        dk[e] = fmaf(ds, chan(q, e), dk[e]);
      }
    }, [&] { return (want_k && !all_nan(dk)) || (want_v && !all_nan(dv)); });
  }
#pragma unroll
  for (int e = 0; e < C; ++e) dk[e] *= a.scale;
  if (want_k) chan_store<C>((bf16*)a.dk + (size_t)kr * a.lddk + (size_t)hk * D + C * lane, dk);
  if (want_v) chan_store<C>((bf16*)a.dv + (size_t)kr * a.lddv + (size_t)hk * D + C * lane, dv);
}
template <int D>
__global__ void __launch_bounds__(256) k_gat_again(const __grid_constant__ Seqs s, const __grid_constant__ AttnArgs a,
                                                   const __grid_constant__ TcArgs tq, const __grid_constant__ TcArgs tk) {
  pdl_launch_dependents();
  pdl_wait();
  if (*a.any == 0) return;
  const int keys = s.kv0[s.B];
  for (long long i = blockIdx.x; i < 16 * (tq.lots + tk.lots); i += gridDim.x) {
    const bool of_keys = i >= 16 * tq.lots;
    const TcArgs& t = of_keys ? tk : tq;
    const long long lot = (of_keys ? i - 16 * tq.lots : i) / 4;
    uint32_t bad[2] = {0, 0};
    if (of_keys) {
      for (int e = 0; e < 8 * tk.parts; ++e) bad[e & 1] |= tk.bad[lot * 8 * tk.parts + e];
    } else {
      for (int e = 0; e < 4 * tq.splits; ++e) bad[0] |= tq.bad[lot * 4 * tq.splits + e];
    }
    const int e = 8 * (int)(i & 3) + (threadIdx.x >> 5);
    const uint32_t bit = 1u << e;
    if (!((bad[0] | bad[1]) & bit)) continue;
    const Where w = t.where[lot];
    // (after a wait that ran out the words are whatever memory held)
    const long long row = w.row + (long long)e * w.step;
    if (row < 0 || row >= (of_keys ? keys : a.rows) || w.head < 0 || w.head >= (of_keys ? a.n_kv : a.n_heads)) continue;
    if (of_keys) key_again<D>(s, a, (int)row, w.head, bad[0] & bit, bad[1] & bit);
    else row_again<D>(s, a, (int)row, w.head);
  }
}

// ---- host ------------------------------------------------------------------------------------------------
// Tiles of the sequences, numbered; returns how many.
int query_tiles(Seqs& s) {
  s.tile0[0] = 0;
  for (int b = 0; b < s.B; ++b) s.tile0[b + 1] = s.tile0[b] + div_up(s.groups[b], groups_per_tile(kT, s.R));
  return s.tile0[s.B];
}
int key_tiles(Seqs& s) {
  s.tile0[0] = 0;
  for (int b = 0; b < s.B; ++b) s.tile0[b + 1] = s.tile0[b] + div_up(s.ctx[b], kT) + div_up(s.groups[b], kT);
  return s.tile0[s.B];
}
// Key tiles of the longest query tile, steps of the key tile that most rows see.
int most_keys(const Seqs& s) {
  int n = 0;
  for (int b = 0; b < s.B; ++b)
    if (s.groups[b]) n = std::max(n, div_up(s.ctx[b], kT) + div_up(s.groups[b], kT) + (s.R > 1));
  return n;
}
int most_steps(const Seqs& s, int per) {
  int n = 0;
  for (int b = 0; b < s.B; ++b) n = std::max(n, div_up(s.groups[b] * s.R, kT) * per);
  return n;
}
// The sequences by length, the longest ones last or first: query tiles are dealt out from the last one's end (the longest
// rows), key tiles from the first one's beginning (those that most rows see).
Seqs sorted(const Seqs& s, bool longest_first) {
  int at[PS_MAX_BATCH];
  for (int b = 0; b < s.B; ++b) at[b] = b;
  std::sort(at, at + s.B, [&](int x, int y) {
    const int kx = div_up(s.ctx[x], kT) + div_up(s.groups[x], kT), ky = div_up(s.ctx[y], kT) + div_up(s.groups[y], kT);
    return kx != ky ? (kx < ky) != longest_first : x < y;
  });
  Seqs r = s;
  for (int b = 0; b < s.B; ++b) {
    r.ctx[b] = s.ctx[at[b]]; r.groups[b] = s.groups[at[b]];
    r.q0[b] = s.q0[at[b]]; r.kv0[b] = s.kv0[at[b]];
  }
  return r;
}

template <class Kern>
cudaError_t ready(Kern kern, int smem, std::atomic<uint64_t>& done) { return allow_smem((const void*)kern, smem, done); }

template <int D>
cudaError_t forward(const Maps& maps, const Seqs& s0, const AttnArgs& a, const TcArgs& t, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (cudaError_t e = ready(k_gat_fwd<D>, Fwd<D>::smem, done)) return e;
  Seqs s = sorted(s0, false);
  const unsigned works = (unsigned)query_tiles(s) * a.n_heads * t.splits;
  cudaError_t e = launch_after(k_gat_fwd<D>, dim3(works), dim3(Fwd<D>::threads), Fwd<D>::smem, st, true, maps, s, a, t);
  if (e != cudaSuccess || t.splits == 1) return e;
  const long long units = (long long)a.rows * a.n_heads;
  return launch_after(k_gat_join<D>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, true, a, t);
}
template <int D>
cudaError_t backward(const Maps& maps, const Seqs& s0, const AttnArgs& a, const TcArgs& tq, const TcArgs& tk, cudaStream_t st) {
  static std::atomic<uint64_t> done_q{0}, done_kv{0};
  if (cudaError_t e = ready(k_gat_dq<D>, Dq<D>::smem, done_q)) return e;
  if (cudaError_t e = ready(k_gat_dkv<D>, Dkv<D>::smem, done_kv)) return e;
  cudaError_t e = cudaSuccess;
  const unsigned sms = device_sms();
  if (a.rows > 0) {
    const int groups = a.rows / s0.R;
    Seqs f = s0;
    f.tile0[0] = 0;
    for (int b = 0; b < f.B; ++b) f.tile0[b + 1] = f.tile0[b] + few_groups(f.ctx[b], f.groups[b]) * f.R;
    if (const int few = f.tile0[f.B]) {
      e = launch_after(k_gat_few<D>, dim3(div_up(few * a.n_heads, 8)), dim3(256), 0, st, true, f, a);
      if (e != cudaSuccess) return e;
    }
    // (registers hold as many rows as a group may have)
    const dim3 blocks((unsigned)(((long long)groups * a.n_kv + 3) / 4));
    if (s0.R == 1) e = launch_after(k_gat_masks<D, 1>, blocks, dim3(128), 0, st, true, s0, a, groups);
    else if (s0.R <= 3) e = launch_after(k_gat_masks<D, 3>, blocks, dim3(128), 0, st, true, s0, a, groups);
    else if (s0.R <= 5) e = launch_after(k_gat_masks<D, 5>, blocks, dim3(128), 0, st, true, s0, a, groups);
    else if (s0.R <= 9) e = launch_after(k_gat_masks<D, 9>, blocks, dim3(128), 0, st, true, s0, a, groups);
    else e = launch_after(k_gat_masks<D, 16>, blocks, dim3(128), 0, st, true, s0, a, groups);
    if (e != cudaSuccess) return e;
    Seqs s = sorted(s0, false);
    const long long works = (long long)query_tiles(s) * a.n_heads * tq.splits;
    e = launch_after(k_gat_dq<D>, dim3((unsigned)std::min<long long>(works, sms)), dim3(Dq<D>::threads), Dq<D>::smem, st, true, maps,
                     s, a, tq);
    if (e == cudaSuccess && tq.splits > 1) {
      const long long units = (long long)a.rows * a.n_heads;
      e = launch_after(k_gat_dq_join<D>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, true, a, tq);
    }
    if (e != cudaSuccess) return e;
  }
  Seqs s = sorted(s0, true);
  const long long tiles = key_tiles(s), works = tiles * a.n_kv * tk.parts;
  e = launch_after(k_gat_dkv<D>, dim3((unsigned)std::min<long long>(works, sms)), dim3(Dkv<D>::threads), Dkv<D>::smem, st, true, maps, s, a, tk);
  if (e == cudaSuccess && tk.parts > 1)
    e = launch_after(k_gat_dkv_join<D>, dim3((unsigned)(tiles * a.n_kv), kT / 16), dim3(256), 0, st, true, s, a, tk);
  if (e != cudaSuccess || a.rows == 0) return e;
  return launch_after(k_gat_again<D>, dim3(2 * sms), dim3(256), 0, st, true, s0, a, tq, tk);
}

}  // namespace

// Parts that a query tile's keys are dealt to, so that few query tiles still fill the device: as many as find room at
// once (two blocks an SM forward, one backward), none with less than two key tiles.
int attn_splits(const Seqs& s, int n_heads, bool backward) {
  Seqs c = s;
  const long long units = (long long)query_tiles(c) * n_heads, room = (backward ? 1 : 2) * device_sms();
  if (units == 0) return 1;
  return std::max(1, (int)std::min<long long>(std::min<long long>(room / units, most_keys(s) / 2), 32));
}
// Parts that a key tile's steps are dealt to, at most kParts: four units of work an SM, so that the last ones end at about
// the same time although the first tiles of a sequence are seen by the most rows.
void attn_parts(const Seqs& s, int n_kv, int per, TcArgs* t) {
  constexpr int kParts = 8;
  Seqs c = s;
  const long long units = (long long)key_tiles(c) * n_kv;
  const int steps = most_steps(s, per);
  t->parts = units == 0 ? 1 : (int)std::max<long long>(1, std::min<long long>(std::min<long long>(kParts, 4ll * device_sms() / units), steps / 4));
  t->cap = std::max(1, div_up(steps, t->parts));
  t->key_units = units * t->parts;
  t->lots = units;
}
long long attn_lots(const Seqs& s, int n_heads) {
  Seqs c = s;
  return (long long)query_tiles(c) * n_heads;
}

bool attn_tc_takes(const AttnArgs& a, bool backward) {
  auto fits = [](const void* p, size_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld < (1ull << 34); };
  if (!(a.scale > 0.f)) return false;
  if (!fits(a.q, a.ldq) || !fits(a.k, a.ldk) || !fits(a.v, a.ldv) || !fits(a.out, a.ldo)) return false;
  return !backward || (fits(a.dout, a.lddo) && fits(a.dq, a.lddq) && fits(a.dk, a.lddk) && fits(a.dv, a.lddv));
}

cudaError_t attn_tc(int D, bool backward_, const Seqs& s, const AttnArgs& a, const TcArgs& t, const TcArgs& tk, cudaStream_t st) {
  Maps m = {};
  const size_t wq = (size_t)a.n_heads * D, wk = (size_t)a.n_kv * D, keys = s.kv0[s.B];
  bool ok = make_rows_map(&m.q, a.q, a.rows, wq, a.ldq, 1) && make_rows_map(&m.k, a.k, keys, wk, a.ldk, 1) &&
            make_rows_map(&m.v, a.v, keys, wk, a.ldv, 1);
  // (a call with fewer rows than a group has no group)
  if (ok && s.R > 1 && keys >= (size_t)s.R)
    ok = make_rows_map(&m.ks, a.k, keys, wk, a.ldk, s.R) && make_rows_map(&m.vs, a.v, keys, wk, a.ldv, s.R);
  if (ok && backward_) ok = make_rows_map(&m.dout, a.dout, a.rows, wq, a.lddo, 1);
  if (!ok) return cudaErrorNotSupported;
  if (backward_) return D == 64 ? backward<64>(m, s, a, t, tk, st) : backward<128>(m, s, a, t, tk, st);
  return D == 64 ? forward<64>(m, s, a, t, st) : forward<128>(m, s, a, t, st);
}

cudaError_t attn_take_status(int* word, cudaStream_t st) { return take_word(word, st); }
cudaError_t attn_wait_expires(long long limit, int* status, cudaStream_t st) { return wait_expires(limit, status, st); }

}  // namespace train
}  // namespace ps
