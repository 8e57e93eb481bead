// sample_rows_f16.cu -- erc_sample_rows' kernels for float16 scores
#include "sample_rows.cuh"

namespace erc {
template erc_status launch_rows<__half>(int64_t, int64_t, const __half*, int64_t, const uint64_t*,
                                     const erc_sample_rule&, int32_t*, float*, int32_t*, cudaStream_t);
}  // namespace erc
