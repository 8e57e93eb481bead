// expert_ffn_tc.cu -- the tensor cores' products for bfloat16, and the tensor maps of both types.
#include <atomic>

#include "expert_ffn_tc.cuh"

namespace erc {

bool tc_encode(CUtensorMap* map, bool bf16, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
               const uint32_t* box) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> entry{nullptr};
  void* f = entry.load();
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || !f)
      return false;
    entry.store(f);
  }
  cuuint64_t d[5], st[4];
  cuuint32_t bx[5], one[5];
  for (int i = 0; i < rank; ++i) d[i] = dims[i], bx[i] = box[i], one[i] = 1;
  for (int i = 0; i + 1 < rank; ++i) st[i] = strides[i];
  return reinterpret_cast<Encode>(f)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
                                     const_cast<void*>(base), d, st, bx, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

ERC_FFN_TC_PRODUCTS(__nv_bfloat16)

}  // namespace erc
