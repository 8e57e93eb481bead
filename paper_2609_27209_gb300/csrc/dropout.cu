// dropout.cu -- dropout from a counter-based generator, with the residual's addition: the mask is a
// function of (key, entry) and never stored, so the gradient is the same kernel.
//
// An entry's word is one of the four of its Philox block.  A thread takes two pieces of 16 bytes of
// each array, one block of the generator a piece for float32 and two for the 16-bit types.
//
// 169343 x 512 bf16 with a residual: 76 to 80 us, 0.96 to 1.01 of the copy rate.  Without one the 16-bit types are bound by
// the generator's instructions on the half-rate integer units: 20000 x 1001 f16 takes 19 us for a floor of 11.8 (blocks of
// 256 threads 19.9, one piece a thread 20.9, four 22.5).
#include "choice.cuh"

namespace erc {
namespace {

constexpr int DT = 128;
constexpr uint32_t DROP = 0x44524F50u;

struct DropRule {
  uint32_t most;  // words up to it are dropped
  bool all;       // everything stays: p below 2^-32 (most is 0 then, and no words are drawn)
  float scale;
  uint64_t key, first;  // first: of the call's first entry, in blocks of 4
};

template <class T>
__device__ __forceinline__ T drop_one(T x, const T* residual, bool keep, const DropRule& d) {
  float v = keep ? __fmul_rn(to_f32(x), d.scale) : 0.f;
  if (residual) v = __fadd_rn(v, to_f32(*residual));
  return from_f32<T>(v);
}

// BLOCKS of the generator at once, from counter `block` on
template <int BLOCKS>
__device__ __forceinline__ void drop_words(uint64_t block, uint64_t key, uint32_t* w) {
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const uint64_t at = block + b;
    const uint4 q = philox4x32_10(make_uint4((uint32_t)at, (uint32_t)(at >> 32), DROP, 0u),
                                  make_uint2((uint32_t)key, (uint32_t)(key >> 32)));
    w[4 * b] = q.x, w[4 * b + 1] = q.y, w[4 * b + 2] = q.z, w[4 * b + 3] = q.w;
  }
}

// a piece of 16 bytes, the first entry's words in w
template <class T, bool RESIDUAL>
__device__ __forceinline__ uint4 drop_piece(uint4 x, uint4 r, const uint32_t* w, const DropRule& d) {
  uint32_t v[4] = {x.x, x.y, x.z, x.w};
  const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      float f = w[i] > d.most ? __fmul_rn(__uint_as_float(v[i]), d.scale) : 0.f;
      if (RESIDUAL) f = __fadd_rn(f, __uint_as_float(q[i]));
      v[i] = __float_as_uint(f);
    } else {
      float2 f = unpack_pair(v[i], T());
      f.x = w[2 * i] > d.most ? __fmul_rn(f.x, d.scale) : 0.f;
      f.y = w[2 * i + 1] > d.most ? __fmul_rn(f.y, d.scale) : 0.f;
      if (RESIDUAL) {
        const float2 g = unpack_pair(q[i], T());
        f.x = __fadd_rn(f.x, g.x);
        f.y = __fadd_rn(f.y, g.y);
      }
      v[i] = pack_pair(f.x, f.y, T());
    }
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// all arrays are 16-byte aligned; a block takes 2 DT pieces of 16 bytes, the last block perhaps fewer
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(DT) k_dropout(int64_t count, const T* x, const T* residual, DropRule d,
                                                const uint64_t* key_dev, T* out) {
  if (key_dev) d.key = *key_dev;
  constexpr int N = 16 / sizeof(T);
  const int64_t from = (int64_t)blockIdx.x * (2 * DT * N) + threadIdx.x * N;  // the thread's entries: N here, N from DT N on
  const uint64_t block = d.first + (uint64_t)from / 4;
  x += from;
  out += from;
  if (RESIDUAL) residual += from;
  if (((int64_t)blockIdx.x + 1) * (2 * DT * N) <= count) {
    uint4 a[2], r[2] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      a[j] = reinterpret_cast<const uint4*>(x)[j * DT];
      if (RESIDUAL) r[j] = reinterpret_cast<const uint4*>(residual)[j * DT];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t w[N];
      if (d.all) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = ~0u;
      } else {
        drop_words<N / 4>(block + j * (DT * N / 4), d.key, w);
      }
      reinterpret_cast<uint4*>(out)[j * DT] = drop_piece<T, RESIDUAL>(a[j], r[j], w, d);
    }
    return;
  }
#pragma unroll 1
  for (int j = 0; j < 2; ++j) {
    uint32_t w[N];
    drop_words<N / 4>(block + j * (DT * N / 4), d.key, w);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = j * DT * N + i;
      if (from + at < count) out[at] = drop_one(x[at], RESIDUAL ? residual + at : nullptr, d.all || w[i] > d.most, d);
    }
  }
}

// four entries a thread, arrays of any alignment
template <class T>
__global__ void __launch_bounds__(DT) k_dropout_any(int64_t count, const T* x, const T* residual, DropRule d,
                                                    const uint64_t* key_dev, T* out) {
  if (key_dev) d.key = *key_dev;
  const int64_t v = (int64_t)blockIdx.x * DT + threadIdx.x;
  if (v * 4 >= count) return;
  uint32_t w[4];
  drop_words<1>(d.first + (uint64_t)v, d.key, w);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t e = v * 4 + i;
    if (e < count) out[e] = drop_one(x[e], residual ? residual + e : nullptr, d.all || w[i] > d.most, d);
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
  ERC_REQUIRE(count >= 0 && count <= (1LL << 40), "count must be in [0, 2^40]");
  ERC_REQUIRE(p >= 0. && p <= 1., "p must be in [0, 1]");
  ERC_REQUIRE(first >= 0 && first % 4 == 0, "first must be a multiple of 4, at least 0");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(key_dev) % 8 == 0, "misaligned key_dev");
  if (count == 0) return ERC_OK;
  ERC_REQUIRE(x && out, "null pointer");
  const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(residual) |
                        reinterpret_cast<uintptr_t>(out);
  ERC_REQUIRE(all % type_bytes(type) == 0, "misaligned x, residual or out");
  const uint64_t least = (uint64_t)(p * 4294967296.);
  DropRule d;
  d.all = least == 0;
  d.most = d.all ? 0u : (uint32_t)(least - 1);
  d.scale = p < 1. ? (float)(1. / (1. - p)) : 0.f;
  d.key = key;
  d.first = (uint64_t)first / 4;
  const cudaStream_t s = as_stream(stream);
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const T *a = static_cast<const T*>(x), *r = static_cast<const T*>(residual);
    T* o = static_cast<T*>(out);
    const bool whole = all % 16 == 0;
    const int64_t each = whole ? 2 * DT * (16 / (int)sizeof(T)) : 4 * DT;
    const unsigned grid = (unsigned)((count + each - 1) / each);
    auto kernel = !whole ? k_dropout_any<T> : r ? k_dropout<T, true> : k_dropout<T, false>;
    kernel<<<grid, DT, 0, s>>>(count, a, r, d, key_dev, o);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
