// sample_rows.cu -- erc_sample_rows: one exact draw per row of scores (sample_rows.cuh)
#include "choice.cuh"

namespace erc {
template <class T>
erc_status launch_rows(int64_t rows, int64_t n, const T* logits, int64_t stride,
                       const uint64_t* words, const erc_sample_rule& rule, int32_t* ids,
                       float* logp, int32_t* kept, cudaStream_t s);
}  // namespace erc

using namespace erc;

extern "C" erc_status erc_sample_rows(int64_t rows, int64_t n, const void* logits, int32_t type,
                                      int64_t stride, const uint64_t* words,
                                      const erc_sample_rule* rule, int32_t* ids, float* logp,
                                      int32_t* kept, erc_stream stream) {
  clear_error();
  ERC_REQUIRE(rows >= 0 && rows <= 0x7fffffffLL, "rows must be in [0, 2^31)");
  ERC_REQUIRE(n >= 0 && n <= ERC_SAMPLE_ROWS_MAX_N, "n must be in [0, 2^22]");
  ERC_REQUIRE(type >= ERC_F32 && type <= ERC_F16, "bad score type %d", type);
  ERC_REQUIRE(stride >= 0, "stride must be >= 0");
  ERC_REQUIRE(rule, "rule is required");
  ERC_REQUIRE(rule->temperature >= 0.f && rule->temperature <= 3.4028234e38f,
              "temperature must be finite and >= 0");
  ERC_REQUIRE(rule->top_p > 0.f && rule->top_p <= 1.f, "top_p must be in (0, 1]");
  ERC_REQUIRE(rule->min_p >= 0.f && rule->min_p <= 1.f, "min_p must be in [0, 1]");
  ERC_REQUIRE(rule->top_k >= 0, "top_k must be >= 0");
  if (rows == 0) return ERC_OK;
  ERC_REQUIRE((logits || n == 0) && words && ids && logp && kept, "null pointer");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(logits) % type_bytes(type) == 0, "misaligned logits");
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    return launch_rows<T>(rows, n, static_cast<const T*>(logits), stride, words, *rule, ids, logp,
                          kept, as_stream(stream));
  });
}
