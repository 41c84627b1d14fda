// Boxes of bf16 rows by TMA, and the products of bf16 tiles, for the attention kernels that take q (and k, v) as they lie in memory.
#pragma once

#include "kv_attention_tc.cuh"

namespace vscan {
namespace kv {

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(tc::smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
// bf16 x bf16 -> float32, M = 128; b_mn: the second operand MN-major
__device__ __forceinline__ uint32_t idesc_bf16(int n, bool b_mn) { return idesc_f16(n, b_mn) | (1u << 7) | (1u << 10); }

// Boxes of 64 channels x `inner` x `outer` of a tensor of sizes[0] x sizes[1] rows by steps (in elements), `batch` of them seq_step apart.  False where
// TMA does not take the strides: heads or rows on top of each other, for one
inline bool rows_map(const void* at, int head_dim, const int64_t (&sizes)[2], const int64_t (&steps)[2], int64_t batch, int64_t seq_step, int inner,
                     int outer, CUtensorMap* map) {
  const auto encode = tc::encode_fn();
  if (!encode) return false;
  const int64_t all[3] = {sizes[0], sizes[1], batch}, step[3] = {steps[0], steps[1], seq_step};
  cuuint64_t dims[4] = {static_cast<cuuint64_t>(head_dim)}, strides[3];
  for (int i = 0; i < 3; ++i) {
    if (all[i] > 1 && step[i] == 0) return false;
    dims[i + 1] = static_cast<cuuint64_t>(all[i]);
    strides[i] = all[i] > 1 ? static_cast<cuuint64_t>(step[i]) * 2 : 16;
  }
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(inner), static_cast<cuuint32_t>(outer), 1}, each[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(at), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace kv
}  // namespace vscan
