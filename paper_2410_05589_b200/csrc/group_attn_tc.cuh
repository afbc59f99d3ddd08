// Interface of the tensor-core attention under the mask of parallel groups (group_attn_tc.cu).
#pragma once
#include "group_attn.cuh"

namespace ps {
namespace train {

struct Maps {
  CUtensorMap q, k, v, ks, vs, dout;   // ks, vs: rows of a group side by side (keys of the second kind)
};
struct TcArgs {
  int splits;         // parts that a query tile's keys are dealt to
  float* part_o;      // [splits][n_heads][rows][D] their outputs (forward) or dq
  float* part_l;      // [splits][n_heads][rows] their log-sum-exps
};

// bf16 rows of `cols` values, ld apart, as [rows / R][R][cols]: boxes of 64 columns and 128 rows that are R apart
// (tensor_map.cu).
bool make_rows_map(CUtensorMap* m, const void* base, size_t rows, size_t cols, size_t ld, int R);
int attn_splits(const Seqs& s, int n_heads, bool backward);
// Whether the tensor maps and vector stores take these pointers and strides (and the softmax its scale: a
// maximum of scores is one of scaled scores).
bool attn_tc_takes(const AttnArgs& a, bool backward);
cudaError_t attn_tc(int D, bool backward, const Seqs& s, const AttnArgs& a, const TcArgs& t, cudaStream_t st);

}  // namespace train
}  // namespace ps
