// sample_rows_bf16.cu -- erc_sample_rows' kernels for bfloat16 scores
#include "sample_rows.cuh"

namespace erc {
template erc_status launch_rows<__nv_bfloat16>(int64_t, int64_t, const __nv_bfloat16*, int64_t, const uint64_t*,
                                     const erc_sample_rule&, int32_t*, float*, int32_t*, cudaStream_t);
}  // namespace erc
