// Interface of the tensor-core attention under the mask of parallel groups (group_attn_tc.cu).
#pragma once
#include "group_attn.cuh"

namespace ps {
namespace train {

struct Maps {
  CUtensorMap q, k, v, ks, vs, dout;   // ks, vs: rows of a group side by side (keys of the second kind)
};
struct Where { int row, step, head; };   // first of 32 rows, rows from one to the next
struct TcArgs {
  int gpt;            // groups of a query tile
  int splits;         // parts that a query tile's keys are dealt to
  float none;         // forward: what a sum of nothing leaves of its outputs, 0 in a part, no number where there is one part
  int parts, cap;     // parts that a key tile's steps are dealt to, steps of a part
  long long key_units;   // key tiles times key heads times parts
  float* part_o;      // [splits][n_heads][rows][D] their outputs (forward) or dq; [key units][dk, dv][128][D]
  float* part_l;      // [splits][n_heads][rows] their log-sum-exps
  // backward: rows (keys) whose sums hold a value that is not finite, a bit each.  For 32 rows of a tile of a head words per
  // part and quarter of the columns (of keys: dk's and dv's), and where the rows lie, written where a word is not 0.
  long long lots;     // tiles times heads
  uint32_t* bad;      // [lots][4][splits or parts][4] ([4][2])
  Where* where;       // [lots][4]
};

// bf16 rows of `cols` values, ld apart, as [rows / R][R][cols]: boxes of 64 columns and 128 rows that are R apart
// (tensor_map.cu).
bool make_rows_map(CUtensorMap* m, const void* base, size_t rows, size_t cols, size_t ld, int R);
int attn_splits(const Seqs& s, int n_heads, bool backward);
void attn_parts(const Seqs& s, int n_kv, int per, TcArgs* t);
long long attn_lots(const Seqs& s, int n_heads);
// Whether the tensor maps and vector stores take these pointers and strides (and the softmax its scale: a
// maximum of scores is one of scaled scores).
bool attn_tc_takes(const AttnArgs& a, bool backward);
cudaError_t attn_tc(int D, bool backward, const Seqs& s, const AttnArgs& a, const TcArgs& t, const TcArgs& tk,
                    cudaStream_t st);   // tk: of the key tiles (backward)

}  // namespace train
}  // namespace ps
