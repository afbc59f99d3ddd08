// Tensor maps of row-major bf16 matrices for tiled TMA.
#include "group_attn_tc.cuh"

namespace ps {
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeTiledFn)p;
  }();
  return fn;
}

}  // namespace

bool make_map(CUtensorMap* m, const void* base, size_t rows, size_t cols, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)cols * 2};
  cuuint32_t box[2] = {(cuuint32_t)kMapCols, (cuuint32_t)box_rows};
  cuuint32_t es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_halves_map(CUtensorMap* m, const void* base, size_t rows, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)kMapCols, (cuuint64_t)rows, 2};
  cuuint64_t strides[2] = {2 * kMapCols * 2, kMapCols * 2};
  cuuint32_t box[3] = {(cuuint32_t)kMapCols, (cuuint32_t)box_rows, 2};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace train {

bool make_rows_map(CUtensorMap* m, const void* base, size_t rows, size_t cols, size_t ld, int R) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn || rows < (size_t)R) return fn && rows == 0;   // (no rows: nothing asks for the map)
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 1};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)R};
  cuuint32_t box[3] = {(cuuint32_t)kMapCols, 128, 1};
  cuuint32_t es[3] = {1, 1, 1};
  if (R > 1) {
    // Groups may begin at any row: a box starts at (row % R, row / R).  Whole multiples of R rows are described; the
    // real row of the last group lies among them, since its masks follow it.
    dims[1] = R;
    dims[2] = rows / R;
    box[1] = 1;
    box[2] = 128;
  }
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, R > 1 ? 3 : 2, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace train
}  // namespace ps
