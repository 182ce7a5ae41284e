// Tensor maps of the operands of q8_linear's tensor-core kernels.  Everything here has internal linkage.
#pragma once
#include "q8_umma_common.cuh"

namespace q8 {
namespace {

constexpr int kMapBlock = 128;  // bytes of the reduction in a block, a swizzle span

// Blocks of the reduction that one load brings.  A load occupies the copy engine for some 370 cycles whatever its size, as
// long as 16 KB take to be multiplied, so two blocks travel together where the row length is whole blocks: the map then
// has the blocks as its third dimension, which cannot cut off a row inside a block.
int blocks_per_load(int C) { return C % kMapBlock == 0 && C > kMapBlock ? 2 : 1; }

// Rows of C bytes `ld` apart, boxes of `box_rows` rows by `blocks` blocks.
int encode_blocks(CUtensorMap* map, const void* base, long long ld, int C, long long rows, int box_rows, int blocks) {
  const DriverFns& fn = driver_fns();
  if (!fn.tiled) return fail(Q8_ERR_CUDA, "q8_linear: cuTensorMapEncodeTiled entry point not available");
  CUresult r;
  const cuuint32_t ones[3] = {1, 1, 1};
  if (blocks > 1) {
    const cuuint64_t dims[3] = {(cuuint64_t)kMapBlock, (cuuint64_t)rows, (cuuint64_t)(C / kMapBlock)}, strides[2] = {(cuuint64_t)ld, (cuuint64_t)kMapBlock};
    const cuuint32_t box[3] = {(cuuint32_t)kMapBlock, (cuuint32_t)box_rows, (cuuint32_t)blocks};
    r = fn.tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else {
    const cuuint64_t dims[2] = {(cuuint64_t)C, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kMapBlock, (cuuint32_t)box_rows};
    r = fn.tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  }
  if (r != CUDA_SUCCESS) return fail(Q8_ERR_CUDA, "q8_linear: tensor map rejected (CUresult %d)", (int)r);
  return Q8_OK;
}

}  // namespace
}  // namespace q8
