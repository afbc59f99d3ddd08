// Input rows of a training step and their gradients (ps_embed_rows, ps_embed_rows_backward).
//
//   out_r = scale * T[id_r],   dT[v] = scale * sum_{r: id_r = v} dout_r
// where T is the token table with the [MASK] rows behind it.
//
// Both are bound by memory.  Forward: a warp per piece of a row, eight 16-byte vectors a lane in flight.
// Backward: the rows are put into the order of their ids (stable: an id's rows increase) and summed from that list in
// pieces of 32 entries, whose sums are added in an order of their own, the same in every call; rows of the table that no id names, most of a large
// vocabulary, are written as zeros meanwhile.
//   k_embed_sort   a block per range of ids reads all of them once (40 KB for 10000 rows: they stay in L2),
//                  counts those below its range, which is where its part of the list begins, and those
//                  in it, per id and eighth of the rows; a second pass puts each eighth's rows in order.  No
//                  block waits for another.  Then it writes its zero rows.
//   k_embed_sum    a block per 32 entries of the list and run of columns; sums in single precision, in the rows' order.  An id
//                  whose rows all lie in the block is stored, the ends of longer ones become partial sums.
//   k_embed_join   adds the partial sums of an id that crosses blocks: every eighth of those behind its first, then
//                  the first and the eight sums.  Where the pieces begin depends on how many rows lower ids have
//                  (a [MASK] row's gradient may differ in its last bits with and without the table's).
// [MASK] ids name a row of every group (thousands of rows each): pieces of 32 keep them from being one
// block's work.
// Measured (with the launches' gaps): 10235 rows of 4096 bf16 forward 26 us (3.9 TB/s; most rows are [MASK] rows that come from
// L2, so that it is the writes); forward and the whole gradient of a table of 128256 x 4096, 10140 rows, 233 us (5.3
// TB/s), of which the zeros take 173 (6.0 TB/s); the [MASK] gradients alone, 2547 rows of 5120, with the forward 31 us,
// which is four launches' latency.  Sixteen rows of a block in flight instead of eight made the table's gradient 249 us.
#include "train_ops.cuh"

namespace ps {
namespace train {
namespace {

constexpr int kWarps = 8;
constexpr int kSlice = 32;         // entries of the list per block of k_embed_sum
constexpr int kMaxRange = 1024;    // ids per block of k_embed_sort
constexpr int kInFlight = 8;

template <class T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N elements that travel together: 16 bytes where pointers, strides and widths allow it, else one element.
template <class T, int N>
struct alignas(sizeof(T) * N) Vec { T v[N]; };

template <class T, int N>
__global__ void __launch_bounds__(32 * kWarps) k_embed_fwd(int rows, int H, int V, int K, const int* __restrict__ ids,
                                                            const T* __restrict__ table, const T* __restrict__ masks,
                                                            float scale, T* __restrict__ out, size_t ldo, int pieces) {
  using P = Vec<T, N>;
  const int nv = H / N, lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (unit >= (long long)rows * pieces) return;
  const int r = (int)(unit / pieces), c0 = (int)(unit - (long long)r * pieces) * 32 * kInFlight + lane;
  const int id = ids[r];
  const T* src = nullptr;
  if (id >= 0 && id < V) src = table + (size_t)id * H;
  else if (id >= V && id < V + K) src = masks + (size_t)(id - V) * H;
  P* dst = reinterpret_cast<P*>(out + (size_t)r * ldo);
  P x[kInFlight];
#pragma unroll
  for (int i = 0; i < kInFlight; ++i) {
    const int c = c0 + 32 * i;
#pragma unroll
    for (int e = 0; e < N; ++e) x[i].v[e] = from_f<T>(0.f);
    if (src && c < nv) x[i] = reinterpret_cast<const P*>(src)[c];
  }
#pragma unroll
  for (int i = 0; i < kInFlight; ++i) {
    const int c = c0 + 32 * i;
    if (c < nv) {
      if (src) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[i].v[e] = from_f<T>(scale * to_f(x[i].v[e]));
      }
      dst[c] = x[i];
    }
  }
}

// An entry of the sorted list: the row, its id, and where the entries of that id begin and end.
struct Entry { int row, id, begin, end; };

struct SortArgs {
  int rows, V, K;
  int lo, hi;          // the ids whose gradients are formed
  int n_tab, range;    // blocks over the table's ids, ids of each; then a block per [MASK] id
  const int* ids;
  Entry* list;
  int* n_list;
};

template <class T, int N>
__global__ void __launch_bounds__(32 * kWarps) k_embed_sort(SortArgs a, int H, T* d_table, T* d_mask) {
  extern __shared__ int s_cnt[];             // [kWarps][range], then [range] begin and [range] end
  __shared__ int s_below[kWarps], s_scan[kWarps];
  __shared__ int s_first;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.x;
  pdl_launch_dependents();
  int v0, v1;
  if (b < a.n_tab) { v0 = b * a.range; v1 = min(a.V, v0 + a.range); }
  else { v0 = a.V + b - a.n_tab; v1 = v0 + 1; }
  const int n = v1 - v0;
  if (n <= 0) return;
  int *s_begin = s_cnt + kWarps * n, *s_end = s_begin + n;
  for (int i = tid; i < kWarps * n; i += 32 * kWarps) s_cnt[i] = 0;
  __syncthreads();
  pdl_wait();      // (the list may still be read by the call before this one)
  // ---- count: warp w has the w-th eighth of the rows
  const int r0 = (int)((long long)a.rows * warp / kWarps), r1 = (int)((long long)a.rows * (warp + 1) / kWarps);
  int below = 0;
  for (int r = r0 + lane; r < r1; r += 32 * 4) {
    int id[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) id[i] = r + 32 * i < r1 ? a.ids[r + 32 * i] : -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      below += id[i] >= a.lo && id[i] < v0;
      if (id[i] >= v0 && id[i] < v1) atomicAdd(&s_cnt[warp * n + id[i] - v0], 1);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) below += __shfl_xor_sync(0xffffffffu, below, o);
  if (lane == 0) s_below[warp] = below;
  __syncthreads();
  if (tid == 0) {
    int s = 0;
    for (int w = 0; w < kWarps; ++w) s += s_below[w];
    s_first = s;
  }
  __syncthreads();
  // ---- where each (id, warp) begins: ids in order, within an id the warps in order
  int at = s_first;
  for (int i0 = 0; i0 < n; i0 += 32 * kWarps) {
    const int i = i0 + tid;
    int total = 0;
    if (i < n)
      for (int w = 0; w < kWarps; ++w) total += s_cnt[w * n + i];
    int inc = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) s_scan[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += s_scan[w];
      all += s_scan[w];
    }
    int p = at + before + inc - total;
    if (i < n) {
      s_begin[i] = p;
      s_end[i] = p + total;
      for (int w = 0; w < kWarps; ++w) {
        const int c = s_cnt[w * n + i];
        s_cnt[w * n + i] = p;
        p += c;
      }
    }
    at += all;
    __syncthreads();
  }
  if (tid == 0 && v1 == a.hi) *a.n_list = at;
  // ---- the list: each warp goes through its rows in order
  if (at > s_first) {
    for (int r = r0; r < r1; r += 32 * 4) {
      int id[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) id[i] = r + 32 * i + lane < r1 ? a.ids[r + 32 * i + lane] : -1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = id[i] >= v0 && id[i] < v1;
        if (__any_sync(0xffffffffu, in)) {
          const unsigned same = __match_any_sync(0xffffffffu, in ? id[i] : -1);
          int p = 0;
          const int leader = __ffs(same) - 1;
          if (in && lane == leader) {
            p = s_cnt[warp * n + id[i] - v0];
            s_cnt[warp * n + id[i] - v0] = p + __popc(same);
          }
          p = __shfl_sync(0xffffffffu, p, leader);
          if (in)
            a.list[p + __popc(same & ((1u << lane) - 1))] =
                Entry{r + 32 * i + lane, id[i], s_begin[id[i] - v0], s_end[id[i] - v0]};
          __syncwarp();
        }
      }
    }
  }
  // ---- ids without a row
  using P = Vec<T, N>;
  P z;
#pragma unroll
  for (int e = 0; e < N; ++e) z.v[e] = from_f<T>(0.f);
  for (int i = warp; i < n; i += kWarps) {
    if (s_end[i] > s_begin[i]) continue;
    T* dst = v0 + i < a.V ? d_table + (size_t)(v0 + i) * H : d_mask + (size_t)(v0 + i - a.V) * H;
    for (int c = lane; c < H / N; c += 32) reinterpret_cast<P*>(dst)[c] = z;
  }
}

template <class T, int N>
__device__ __forceinline__ void store_grad(const float (&x)[N], float scale, int id, int V, int H, int col, T* d_table,
                                           T* d_mask) {
  Vec<T, N> y;
#pragma unroll
  for (int e = 0; e < N; ++e) y.v[e] = from_f<T>(scale * x[e]);
  T* dst = id < V ? d_table + (size_t)id * H : d_mask + (size_t)(id - V) * H;
  *reinterpret_cast<Vec<T, N>*>(dst + col) = y;
}
template <int N>
__device__ __forceinline__ void store_part(const float (&x)[N], float* dst) {
#pragma unroll
  for (int e = 0; e < N; ++e) dst[e] = x[e];
}

template <class T, int N>
__global__ void k_embed_sum(int V, int H, const int* n_list, const Entry* __restrict__ list, const T* __restrict__ dout,
                            size_t ldd, float scale, T* d_table, T* d_mask, float* first, float* last) {
  __shared__ Entry s_e[kSlice];
  pdl_launch_dependents();
  pdl_wait();
  const int s0 = blockIdx.x * kSlice, cnt = min(kSlice, *n_list - s0);
  if (cnt <= 0) return;
  if (threadIdx.x < cnt) s_e[threadIdx.x] = list[s0 + threadIdx.x];
  __syncthreads();
  const int col = (blockIdx.y * blockDim.x + threadIdx.x) * N;
  if (col >= H) return;
  using P = Vec<T, N>;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  for (int i0 = 0; i0 < cnt; i0 += kInFlight) {
    P x[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (i0 + i < cnt) x[i] = *reinterpret_cast<const P*>(dout + (size_t)s_e[i0 + i].row * ldd + col);
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (i0 + i >= cnt) break;
      const Entry en = s_e[i0 + i];
      const int p = s0 + i0 + i;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += to_f(x[i].v[e]);
      if (p + 1 == en.end || p + 1 == s0 + cnt) {      // the id's last row, or the block's
        if (en.begin < s0) store_part<N>(acc, first + (size_t)blockIdx.x * H + col);
        else if (en.end > s0 + cnt) store_part<N>(acc, last + (size_t)blockIdx.x * H + col);
        else store_grad<T, N>(acc, scale, en.id, V, H, col, d_table, d_mask);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
      }
    }
  }
}

constexpr int kJoinWays = 8;
// Block (slice, columns): where an id begins in the slice and goes on behind it, its partial sums; kJoinWays
// threads a column, each every kJoinWays-th of them, then their sums one after the other.
template <class T, int N>
__global__ void __launch_bounds__(32 * kJoinWays) k_embed_join(int V, int H, const int* n_list,
                                                                const Entry* __restrict__ list, float scale,
                                                                const float* __restrict__ first,
                                                                const float* __restrict__ last, T* d_table, T* d_mask) {
  __shared__ float s_x[kJoinWays][32][N + 1];
  pdl_wait();
  const int s0 = blockIdx.x * kSlice, end = s0 + kSlice;
  if (end >= *n_list) return;
  const Entry en = list[end - 1];
  if (en.begin < s0 || en.end <= end) return;
  const int tail = (en.end - end + kSlice - 1) / kSlice;   // slices that hold the rest
  const int x = threadIdx.x, y = threadIdx.y, col = (blockIdx.y * 32 + x) * N;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  if (col < H) {
#pragma unroll 4
    for (int t = y; t < tail; t += kJoinWays) {
      const float* f = first + (size_t)(blockIdx.x + 1 + t) * H + col;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) s_x[y][x][e] = acc[e];
  __syncthreads();
  if (y == 0 && col < H) {
    const float* l = last + (size_t)blockIdx.x * H + col;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float s = l[e];
#pragma unroll
      for (int w = 0; w < kJoinWays; ++w) s += s_x[w][x][e];
      acc[e] = s;
    }
    store_grad<T, N>(acc, scale, en.id, V, H, col, d_table, d_mask);
  }
}

struct EmbedBuf { Entry* list; int* n_list; float *first, *last; size_t bytes; };
EmbedBuf embed_carve(void* ws, int rows, int hidden) {
  Carve c(ws);
  const size_t slices = ((size_t)rows + kSlice - 1) / kSlice;
  EmbedBuf b;
  b.n_list = c.take<int>(1);
  b.list = c.take<Entry>(rows);
  b.first = c.take<float>(slices * hidden);
  b.last = c.take<float>(slices * hidden);
  b.bytes = c.at;
  return b;
}

bool sizes_ok(int dtype, int rows, int hidden, int vocab, int k_masks) {
  return (dtype == PS_DTYPE_F32 || dtype == PS_DTYPE_BF16) && rows >= 0 && rows <= (1 << 24) && hidden >= 1 &&
         hidden <= 65536 && vocab >= 1 && vocab <= (1 << 20) && k_masks >= 0 && k_masks <= PS_MAX_MASKS;
}
const char kSizes[] = "ps_embed_rows: dtype 0 or 1, 0 <= rows <= 2^24, 1 <= hidden <= 65536, 1 <= vocab <= 2^20, "
                      "0 <= k_masks <= 15";

template <class T, int N>
cudaError_t embed_fwd(int rows, int H, int V, int K, const int* ids, const void* table, const void* masks, float scale,
                      void* out, size_t ldo, cudaStream_t st) {
  const int pieces = (H / N + 32 * kInFlight - 1) / (32 * kInFlight);
  const long long units = (long long)rows * pieces;
  k_embed_fwd<T, N><<<(unsigned)((units + kWarps - 1) / kWarps), 32 * kWarps, 0, st>>>(
      rows, H, V, K, ids, (const T*)table, (const T*)masks, scale, (T*)out, ldo, pieces);
  return cudaGetLastError();
}

template <class T, int N>
cudaError_t embed_bwd(const SortArgs& a, int H, float scale, const void* dout, size_t ldd, void* d_table, void* d_mask,
                      const EmbedBuf& b, cudaStream_t st) {
  T *dt = (T*)d_table, *dm = (T*)d_mask;
  const int widest = std::max(a.n_tab ? std::min(a.range, a.V) : 1, 1);
  cudaError_t e = launch_after(k_embed_sort<T, N>, dim3(a.n_tab + (d_mask ? a.K : 0)), dim3(32 * kWarps),
                               (size_t)(kWarps + 2) * widest * sizeof(int), st, true, a, H, dt, dm);
  if (e != cudaSuccess || a.rows == 0) return e;
  const unsigned slices = (unsigned)((a.rows + kSlice - 1) / kSlice);
  const int nv = H / N, threads = std::min(256, (nv + 31) / 32 * 32);
  e = launch_after(k_embed_sum<T, N>, dim3(slices, (nv + threads - 1) / threads), dim3(threads), 0, st, true, a.V, H,
                   (const int*)b.n_list, (const Entry*)b.list, (const T*)dout, ldd, scale, dt, dm, b.first, b.last);
  if (e != cudaSuccess || slices < 2) return e;
  return launch_after(k_embed_join<T, N>, dim3(slices - 1, (nv + 31) / 32), dim3(32, kJoinWays), 0, st, true, a.V, H,
                      (const int*)b.n_list, (const Entry*)b.list, scale, (const float*)b.first, (const float*)b.last, dt, dm);
}

}  // namespace
}  // namespace train
}  // namespace ps

using namespace ps;
using namespace ps::train;

extern "C" ps_status ps_embed_rows(int dtype, int rows, int hidden, int vocab, int k_masks, const int* ids,
                                   const void* table, const void* mask_rows, float scale, void* out, size_t ldo,
                                   char* err_text, size_t err_cap, void* stream) {
  const Err err{err_text, err_cap};
  if (err_text && err_cap) err_text[0] = 0;
  if (!sizes_ok(dtype, rows, hidden, vocab, k_masks)) return err(PS_ERR_INVALID_ARG, kSizes);
  if (ldo < (size_t)hidden) return err(PS_ERR_INVALID_ARG, "ps_embed_rows: ldo is smaller than hidden");
  if (rows == 0) return PS_OK;
  if (!ids || !table || !out || (k_masks && !mask_rows)) return err(PS_ERR_INVALID_ARG, "ps_embed_rows: null pointer");
  const size_t es = dtype == PS_DTYPE_F32 ? 4 : 2;
  const bool vec = aligned(table, 16) && aligned(mask_rows, 16) && aligned(out, 16) && hidden * es % 16 == 0 && ldo * es % 16 == 0;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (dtype == PS_DTYPE_F32)
    e = vec ? embed_fwd<float, 4>(rows, hidden, vocab, k_masks, ids, table, mask_rows, scale, out, ldo, st)
            : embed_fwd<float, 1>(rows, hidden, vocab, k_masks, ids, table, mask_rows, scale, out, ldo, st);
  else
    e = vec ? embed_fwd<__nv_bfloat16, 8>(rows, hidden, vocab, k_masks, ids, table, mask_rows, scale, out, ldo, st)
            : embed_fwd<__nv_bfloat16, 1>(rows, hidden, vocab, k_masks, ids, table, mask_rows, scale, out, ldo, st);
  return err.cuda(e, "ps_embed_rows");
}

extern "C" size_t ps_embed_rows_workspace_bytes(int dtype, int rows, int hidden, int vocab, int k_masks) {
  return sizes_ok(dtype, rows, hidden, vocab, k_masks) ? embed_carve(nullptr, rows, hidden).bytes : 0;
}

extern "C" ps_status ps_embed_rows_backward(int dtype, int rows, int hidden, int vocab, int k_masks, const int* ids,
                                            float scale, const void* dout, size_t lddo, void* d_table, void* d_mask,
                                            void* workspace, size_t workspace_bytes, char* err_text, size_t err_cap,
                                            void* stream) {
  const Err err{err_text, err_cap};
  if (err_text && err_cap) err_text[0] = 0;
  if (!sizes_ok(dtype, rows, hidden, vocab, k_masks)) return err(PS_ERR_INVALID_ARG, kSizes);
  if (lddo < (size_t)hidden) return err(PS_ERR_INVALID_ARG, "ps_embed_rows_backward: lddo is smaller than hidden");
  if (k_masks == 0) d_mask = nullptr;
  if (!d_table && !d_mask) return PS_OK;
  if (rows && (!ids || !dout)) return err(PS_ERR_INVALID_ARG, "ps_embed_rows_backward: null pointer");
  const EmbedBuf b = embed_carve(workspace, rows, hidden);
  if (ps_status s = check_workspace(err, "ps_embed_rows_backward", workspace, workspace_bytes, b.bytes)) return s;
  SortArgs a;
  a.rows = rows; a.V = vocab; a.K = k_masks;
  a.lo = d_table ? 0 : vocab;
  a.hi = d_mask ? vocab + k_masks : vocab;
  a.n_tab = 0; a.range = 1;
  if (d_table) {
    const int want = std::max(4 * device_sms(), (vocab + kMaxRange - 1) / kMaxRange);
    a.range = (vocab + want - 1) / want;
    a.n_tab = (vocab + a.range - 1) / a.range;
  }
  a.ids = ids; a.list = b.list; a.n_list = b.n_list;
  const size_t es = dtype == PS_DTYPE_F32 ? 4 : 2;
  const bool vec = aligned(d_table, 16) && aligned(d_mask, 16) && aligned(dout, 16) && hidden * es % 16 == 0 && lddo * es % 16 == 0;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (dtype == PS_DTYPE_F32)
    e = vec ? embed_bwd<float, 4>(a, hidden, scale, dout, lddo, d_table, d_mask, b, st)
            : embed_bwd<float, 1>(a, hidden, scale, dout, lddo, d_table, d_mask, b, st);
  else
    e = vec ? embed_bwd<__nv_bfloat16, 8>(a, hidden, scale, dout, lddo, d_table, d_mask, b, st)
            : embed_bwd<__nv_bfloat16, 1>(a, hidden, scale, dout, lddo, d_table, d_mask, b, st);
  return err.cuda(e, "ps_embed_rows_backward");
}
