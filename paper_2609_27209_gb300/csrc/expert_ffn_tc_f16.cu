// expert_ffn_tc_f16.cu -- the tensor cores' products for float16.
#include "expert_ffn_tc.cuh"

namespace erc {

ERC_FFN_TC_PRODUCTS(__half)

}  // namespace erc
