// Tensor maps of the segment-attention kernels (bf16).
#pragma once
#include "seg_attn.cuh"
#include "tc_ptx.cuh"

namespace swam {
namespace {

bool encode_bf16(CUtensorMap* map, const void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                 CUtensorMapL2promotion fetch = CU_TENSOR_MAP_L2_PROMOTION_L2_256B) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, box[0] == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            fetch, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [blocks, n, N_kv, D] with strides, viewed as (d, row, head, block); box = 64 (head dim 32: 32) columns x box_rows rows
bool make_kv_map(CUtensorMap* map, const void* ptr, int blocks, int n, int N_kv, int D, int64_t tok, int64_t smp, int box_rows,
                 CUtensorMapL2promotion fetch = CU_TENSOR_MAP_L2_PROMOTION_L2_256B) {
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)n, (cuuint64_t)N_kv, (cuuint64_t)blocks};
  const cuuint64_t strides[3] = {(cuuint64_t)tok * 2, (cuuint64_t)D * 2, (cuuint64_t)smp * 2};
  const cuuint32_t box[4] = {(cuuint32_t)(D == 32 ? 32 : 64), (cuuint32_t)box_rows, 1, 1};
  return encode_bf16(map, ptr, 4, dims, strides, box, fetch);
}

}  // namespace
}  // namespace swam
