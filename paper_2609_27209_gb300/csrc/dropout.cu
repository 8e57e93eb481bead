// dropout.cu -- dropout from a counter-based generator, with the residual's addition: the mask is a
// function of (key, entry) and never stored, so the gradient is the same kernel.
//
// An entry's word is one of the four of its Philox block; a thread takes 16 bytes, one block of the
// generator for float32 and two for the 16-bit types.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int DT = 256;
constexpr uint32_t DROP = 0x44524F50u;

struct DropRule {
  uint64_t least;  // floor(p 2^32): smaller words are dropped
  float scale;
  uint64_t key, first;  // first: of the call's first entry, in blocks of 4
};

template <class T>
__device__ __forceinline__ T drop_one(T x, const T* residual, uint32_t word, const DropRule& d) {
  float v = word >= d.least ? __fmul_rn(to_f32(x), d.scale) : 0.f;
  if (residual) v = __fadd_rn(v, to_f32(*residual));
  return from_f32<T>(v);
}

__device__ __forceinline__ uint4 drop_words(uint64_t block, uint64_t key) {
  return philox4x32_10(make_uint4((uint32_t)block, (uint32_t)(block >> 32), DROP, 0u),
                       make_uint2((uint32_t)key, (uint32_t)(key >> 32)));
}

// VEC: all arrays are 16-byte aligned
template <class T, bool VEC>
__global__ void __launch_bounds__(DT) k_dropout(int64_t count, const T* x, const T* residual,
                                                DropRule d, const uint64_t* key_dev, T* out) {
  if (key_dev) d.key = *key_dev;
  constexpr int N = VEC ? 16 / sizeof(T) : 4;
  const int64_t groups = (count + N - 1) / N;
  for (int64_t v = (int64_t)blockIdx.x * DT + threadIdx.x; v < groups; v += (int64_t)gridDim.x * DT) {
    uint32_t w[N];
#pragma unroll
    for (int b = 0; b < N / 4; ++b) {
      const uint4 q = drop_words(d.first + (uint64_t)v * (N / 4) + b, d.key);
      w[4 * b] = q.x, w[4 * b + 1] = q.y, w[4 * b + 2] = q.z, w[4 * b + 3] = q.w;
    }
    if (VEC && (v + 1) * N <= count) {
      union Piece {
        uint4 raw;
        T t[N];
        __device__ Piece() {}
      } a, r;
      a.raw = reinterpret_cast<const uint4*>(x)[v];
      if (residual) r.raw = reinterpret_cast<const uint4*>(residual)[v];
#pragma unroll
      for (int i = 0; i < N; ++i) a.t[i] = drop_one(a.t[i], residual ? &r.t[i] : nullptr, w[i], d);
      reinterpret_cast<uint4*>(out)[v] = a.raw;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t e = v * N + i;
        if (e < count) out[e] = drop_one(x[e], residual ? residual + e : nullptr, w[i], d);
      }
    }
  }
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" erc_status erc_dropout(int64_t count, const void* x, int32_t type, const void* residual,
                                  double p, uint64_t key, const uint64_t* key_dev, int64_t first,
                                  void* out, erc_stream stream) {
  clear_error();
  ERC_REQUIRE(type >= ERC_F32 && type <= ERC_F16, "bad type %d", type);
  ERC_REQUIRE(count >= 0 && count <= (1LL << 48), "count must be in [0, 2^48]");
  ERC_REQUIRE(p >= 0. && p <= 1., "p must be in [0, 1]");
  ERC_REQUIRE(first >= 0 && first % 4 == 0, "first must be a multiple of 4, at least 0");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(key_dev) % 8 == 0, "misaligned key_dev");
  if (count == 0) return ERC_OK;
  ERC_REQUIRE(x && out, "null pointer");
  const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(residual) |
                        reinterpret_cast<uintptr_t>(out);
  ERC_REQUIRE(all % type_bytes(type) == 0, "misaligned x, residual or out");
  DropRule d;
  d.least = (uint64_t)(p * 4294967296.);
  d.scale = p < 1. ? (float)(1. / (1. - p)) : 0.f;
  d.key = key;
  d.first = (uint64_t)first / 4;
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const bool vec = all % 16 == 0;
    const int64_t groups = count / (vec ? 16 / (int)sizeof(T) : 4) + 1;
    const int64_t most = (int64_t)sm_count() * 32;
    const int64_t blocks = (groups + DT - 1) / DT;
    auto kernel = vec ? k_dropout<T, true> : k_dropout<T, false>;
    kernel<<<(unsigned)(blocks < most ? blocks : most), DT, 0, as_stream(stream)>>>(
        count, static_cast<const T*>(x), static_cast<const T*>(residual), d, key_dev,
        static_cast<T*>(out));
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
