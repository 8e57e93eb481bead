// experts.cu -- the chosen (row, choice) pairs in expert order, rows copied into that order, and
// the weighted sum back, with its gradient.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int PT = 256;     // threads of a plan tile
constexpr int PTILE = 1024;  // pairs of a plan tile
constexpr int MAX_E = ERC_ROUTE_MAX_EXPERTS;

struct Plan {
  int32_t* tile;  // [tiles][E] pairs of each expert, then their exclusive sums over tiles
};
void plan_experts(Arena& a, Plan& p, int64_t pairs, int E) {
  p.tile = a.take<int32_t>((size_t)((pairs + PTILE - 1) / PTILE) * E);
}

__global__ void __launch_bounds__(PT) k_plan_count(const int32_t* __restrict__ experts,
                                                   int64_t pairs, int E,
                                                   int32_t* __restrict__ tile) {
  __shared__ int32_t c[MAX_E];
  for (int e = threadIdx.x; e < E; e += PT) c[e] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * PTILE;
  for (int i = threadIdx.x; i < PTILE && base + i < pairs; i += PT) {
    const int e = experts[base + i];
    if (e >= 0 && e < E) atomicAdd(&c[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += PT) tile[(int64_t)blockIdx.x * E + e] = c[e];
}

__global__ void __launch_bounds__(MAX_E) k_plan_scan(int32_t* __restrict__ tile, int tiles, int E,
                                                     int64_t* __restrict__ offsets) {
  __shared__ int32_t total[MAX_E];
  const int e = threadIdx.x;
  int32_t sum = 0;
  if (e < E)
    for (int t = 0; t < tiles; ++t) {
      const int32_t v = tile[(int64_t)t * E + e];
      tile[(int64_t)t * E + e] = sum;
      sum += v;
    }
  total[e] = e < E ? sum : 0;
  __syncthreads();
  if (e == 0) {
    int64_t s = 0;
    for (int i = 0; i < E; ++i) {
      offsets[i] = s;
      s += total[i];
    }
    offsets[E] = s;
  }
}

// a pair's slot: its expert's offset, the pairs of that expert in earlier tiles, and those before
// it in its tile
__global__ void __launch_bounds__(PT) k_plan_place(const int32_t* __restrict__ experts,
                                                   int64_t pairs, int E,
                                                   const int32_t* __restrict__ tile,
                                                   const int64_t* __restrict__ offsets,
                                                   int32_t* __restrict__ order,
                                                   int32_t* __restrict__ slot) {
  __shared__ int32_t next[MAX_E];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t base = (int64_t)blockIdx.x * PTILE;
  for (int e = threadIdx.x; e < E; e += PT)
    next[e] = (int32_t)offsets[e] + tile[(int64_t)blockIdx.x * E + e];
  const int64_t placed = offsets[E];
  for (int i = threadIdx.x; i < PTILE && base + i < pairs; i += PT)
    if (base + i >= placed) order[base + i] = -1;
  __syncthreads();
  for (int g = 0; g < PTILE / 32; ++g) {  // 32 pairs at a time, in order
    if (g % (PT / 32) == warp) {
      const int64_t i = base + g * 32 + lane;
      const int e = i < pairs ? experts[i] : -1;
      const bool some = e >= 0 && e < E;
      const unsigned same = __match_any_sync(0xffffffffu, some ? e : -1);
      int32_t at = 0;
      if (some) at = next[e] + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (some && lane == 31 - __clz(same)) next[e] = at + 1;
      if (some) order[at] = (int32_t)i;
      if (i < pairs) slot[i] = some ? at : -1;
    }
    __syncthreads();
  }
}

template <class T>
__global__ void __launch_bounds__(256) k_combine(int64_t rows, int k, int64_t width,
                                                 const T* __restrict__ y,
                                                 const int32_t* __restrict__ slot,
                                                 const float* __restrict__ weights,
                                                 T* __restrict__ out) {
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x)
    for (int64_t d = threadIdx.x; d < width; d += 256) {
      float s = 0.f;
      for (int j = 0; j < k; ++j) {
        const int32_t p = slot[t * k + j];
        if (p < 0 || p >= rows * k) continue;
        const float v = to_f32(y[p * width + d]);
        s = weights ? fmaf(weights[t * k + j], v, s) : s + v;
      }
      out[t * width + d] = from_f32<T>(s);
    }
}

// dy[slot] = weight * g[row] (weights NULL: a copy) and dweights = g[row] . y[slot]
template <class T>
__global__ void __launch_bounds__(256) k_expand(int64_t rows, int k, int64_t width,
                                                const T* __restrict__ g, const T* __restrict__ y,
                                                const int32_t* __restrict__ slot,
                                                const int64_t* __restrict__ placed,
                                                const float* __restrict__ weights,
                                                T* __restrict__ dy, float* __restrict__ dweights) {
  __shared__ float part[8];
  const int tid = threadIdx.x;
  const int64_t from = *placed < 0 ? 0 : *placed;  // slots without a pair
  for (int64_t u = from + blockIdx.x; u < rows * k; u += gridDim.x)
    for (int64_t d = tid; d < width; d += 256) dy[u * width + d] = from_f32<T>(0.f);
  for (int64_t u = blockIdx.x; u < rows * k; u += gridDim.x) {
    const int32_t p = slot[u];
    const int64_t t = u / k;
    const float w = weights ? weights[u] : 1.f;
    float s = 0.f;
    if (p >= 0 && p < rows * k)
      for (int64_t d = tid; d < width; d += 256) {
        const float v = to_f32(g[t * width + d]);
        dy[p * width + d] = from_f32<T>(weights ? w * v : v);
        if (dweights) s = fmaf(v, to_f32(y[p * width + d]), s);
      }
    if (dweights) {
#pragma unroll
      for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      __syncthreads();
      if ((tid & 31) == 0) part[tid >> 5] = s;
      __syncthreads();
      if (tid == 0) {
        s = 0.f;
        for (int i = 0; i < 8; ++i) s += part[i];
        dweights[u] = s;
      }
    }
  }
}

erc_status check_sizes(int64_t rows, int32_t k, int64_t width, int32_t type) {
  ERC_REQUIRE(type >= ERC_F32 && type <= ERC_F16, "bad type %d", type);
  ERC_REQUIRE(k >= 1 && k <= ERC_ROUTE_MAX_K, "k must be in [1, %d]", ERC_ROUTE_MAX_K);
  ERC_REQUIRE(rows >= 0 && rows <= 0x7fffffffLL / k, "rows * k must be in [0, 2^31)");
  ERC_REQUIRE(width >= 0 && width <= (1LL << 24), "width must be in [0, 2^24]");
  return ERC_OK;
}
bool aligned(const void* p, int32_t type) {
  return reinterpret_cast<uintptr_t>(p) % type_bytes(type) == 0;
}
unsigned row_grid(int64_t rows) {
  const int64_t most = 64LL * sm_count();
  return (unsigned)(rows < most ? rows : most);
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" size_t erc_expert_plan_workspace_size(int64_t rows, int32_t k, int32_t experts) {
  if (rows < 0 || k < 1 || k > ERC_ROUTE_MAX_K || rows > 0x7fffffffLL / k || experts < 1 ||
      experts > MAX_E)
    return 0;
  Arena a(nullptr);
  Plan p;
  plan_experts(a, p, rows * k, experts);
  return a.used + 256;
}

extern "C" erc_status erc_expert_plan(int64_t rows, int32_t k, int32_t n_experts,
                                      const int32_t* experts, int64_t* offsets, int32_t* order,
                                      int32_t* slot, void* ws, size_t ws_bytes, erc_stream stream) {
  clear_error();
  ERC_REQUIRE(k >= 1 && k <= ERC_ROUTE_MAX_K, "k must be in [1, %d]", ERC_ROUTE_MAX_K);
  ERC_REQUIRE(rows >= 0 && rows <= 0x7fffffffLL / k, "rows * k must be in [0, 2^31)");
  ERC_REQUIRE(n_experts >= 1 && n_experts <= MAX_E, "experts must be in [1, %d]", MAX_E);
  ERC_REQUIRE(offsets, "offsets is required");
  cudaStream_t s = as_stream(stream);
  const int64_t pairs = rows * k;
  if (pairs == 0) {
    ERC_CUDA(cudaMemsetAsync(offsets, 0, (n_experts + 1) * sizeof(int64_t), s));
    return ERC_OK;
  }
  ERC_REQUIRE(experts && order && slot, "null pointer");
  if (!ws || ws_bytes < erc_expert_plan_workspace_size(rows, k, n_experts))
    return set_error(ERC_ERR_CAPACITY, "workspace too small");
  Arena ar(reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~uintptr_t(255)));
  Plan p;
  plan_experts(ar, p, pairs, n_experts);
  const unsigned tiles = (unsigned)((pairs + PTILE - 1) / PTILE);
  k_plan_count<<<tiles, PT, 0, s>>>(experts, pairs, n_experts, p.tile);
  k_plan_scan<<<1, MAX_E, 0, s>>>(p.tile, (int)tiles, n_experts, offsets);
  k_plan_place<<<tiles, PT, 0, s>>>(experts, pairs, n_experts, p.tile, offsets, order, slot);
  count_launches(3);
  ERC_CUDA(cudaGetLastError());
  return ERC_OK;
}

extern "C" erc_status erc_expert_combine(int64_t rows, int32_t k, int64_t width, const void* y,
                                         int32_t type, const int32_t* slot, const float* weights,
                                         void* out, erc_stream stream) {
  clear_error();
  ERC_TRY(check_sizes(rows, k, width, type));
  if (rows == 0 || width == 0) return ERC_OK;
  ERC_REQUIRE(y && slot && out, "null pointer");
  ERC_REQUIRE(aligned(y, type) && aligned(out, type), "misaligned y or out");
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    k_combine<T><<<row_grid(rows), 256, 0, as_stream(stream)>>>(
        rows, k, width, static_cast<const T*>(y), slot, weights, static_cast<T*>(out));
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}

namespace {
erc_status expand(int64_t rows, int32_t k, int64_t width, const void* g, const void* y,
                  int32_t type, const int32_t* slot, const int64_t* placed, const float* weights,
                  void* dy, float* dweights, erc_stream stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    k_expand<T><<<row_grid(rows * k), 256, 0, as_stream(stream)>>>(
        rows, k, width, static_cast<const T*>(g), static_cast<const T*>(y), slot, placed, weights,
        static_cast<T*>(dy), dweights);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
}  // namespace

extern "C" erc_status erc_expert_gather(int64_t rows, int32_t k, int64_t width, const void* x,
                                        int32_t type, const int32_t* slot, const int64_t* placed,
                                        void* xs, erc_stream stream) {
  clear_error();
  ERC_TRY(check_sizes(rows, k, width, type));
  if (rows == 0 || width == 0) return ERC_OK;
  ERC_REQUIRE(x && slot && placed && xs, "null pointer");
  ERC_REQUIRE(aligned(x, type) && aligned(xs, type), "misaligned x or xs");
  return expand(rows, k, width, x, nullptr, type, slot, placed, nullptr, xs, nullptr, stream);
}

extern "C" erc_status erc_expert_combine_backward(int64_t rows, int32_t k, int64_t width,
                                                  const void* dout, const void* y, int32_t type,
                                                  const int32_t* slot, const int64_t* placed,
                                                  const float* weights, void* dy, float* dweights,
                                                  erc_stream stream) {
  clear_error();
  ERC_TRY(check_sizes(rows, k, width, type));
  if (rows == 0) return ERC_OK;
  ERC_REQUIRE(slot && placed && weights && dweights, "null pointer");
  if (width == 0) {
    ERC_CUDA(cudaMemsetAsync(dweights, 0, rows * k * sizeof(float), as_stream(stream)));
    return ERC_OK;
  }
  ERC_REQUIRE(dout && y && dy, "null pointer");
  ERC_REQUIRE(aligned(dout, type) && aligned(y, type) && aligned(dy, type),
              "misaligned dout, y or dy");
  return expand(rows, k, width, dout, y, type, slot, placed, weights, dy, dweights, stream);
}
