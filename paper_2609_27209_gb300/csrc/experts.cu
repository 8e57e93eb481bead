// experts.cu -- the chosen (row, choice) pairs in expert order, rows copied into that order, and
// the weighted sum back, with its gradient.
#include <initializer_list>

#include "choice.cuh"

namespace erc {
namespace {

constexpr int PT = 256;        // threads of a plan tile
constexpr int PW = PT / 32;    // its warps
constexpr int PTILE = 2048;    // pairs of a plan tile: a warp takes PTILE / PW consecutive ones
constexpr int MAX_E = ERC_ROUTE_MAX_EXPERTS;

struct Plan {
  int32_t* tile;   // [E][tiles] pairs of each expert, then their exclusive sums over the tiles
  int32_t* total;  // [E]
};
int64_t plan_tiles(int64_t pairs) { return (pairs + PTILE - 1) / PTILE; }
void plan_experts(Arena& a, Plan& p, int64_t pairs, int E) {
  p.tile = a.take<int32_t>((size_t)plan_tiles(pairs) * E);
  p.total = a.take<int32_t>(E);
}

__global__ void __launch_bounds__(PT) k_plan_count(const int32_t* __restrict__ experts,
                                                   int64_t pairs, int E, int tiles,
                                                   int32_t* __restrict__ tile) {
  __shared__ int32_t c[MAX_E];
  for (int e = threadIdx.x; e < E; e += PT) c[e] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * PTILE;
  int mine[PTILE / PT];
#pragma unroll
  for (int j = 0; j < PTILE / PT; ++j) {
    const int64_t i = base + j * PT + threadIdx.x;
    mine[j] = i < pairs ? experts[i] : -1;
  }
#pragma unroll
  for (int j = 0; j < PTILE / PT; ++j)
    if (mine[j] >= 0 && mine[j] < E) atomicAdd(&c[mine[j]], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += PT) tile[(int64_t)e * tiles + blockIdx.x] = c[e];
}

// a block scans an expert's counts over the tiles
__global__ void __launch_bounds__(PT) k_plan_scan(int32_t* __restrict__ tile, int tiles,
                                                  int32_t* __restrict__ total) {
  __shared__ int32_t part[PW];
  int32_t* t = tile + (int64_t)blockIdx.x * tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t before = 0;
  for (int base = 0; base < tiles; base += PT) {
    const int i = base + threadIdx.x;
    const int32_t v = i < tiles ? t[i] : 0;
    int32_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int32_t mine = before;
#pragma unroll
    for (int w = 0; w < PW; ++w) {
      if (w < warp) mine += part[w];
      before += part[w];
    }
    if (i < tiles) t[i] = mine + x - v;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = before;
}

// A pair's slot: its expert's offset, the expert's pairs in earlier tiles, in earlier warps of its
// tile, and before it in its warp.  Every block adds up the experts' totals (one tile: its own).  A
// warp's pairs stay in registers between its counting and its placing, eight loads in flight.
//
// 169,343 x 8 pairs, 256 experts: count, scan and place take 25 to 31 us for 16 MB, 2.4 us of copying.
// One by one with cold caches they take 6, 6 and 18 us; the last waits for its counts, one sector a
// count, and for its 32 pairs after 32.
__global__ void __launch_bounds__(PT) k_plan_place(const int32_t* __restrict__ experts,
                                                   int64_t pairs, int E, int tiles,
                                                   const int32_t* __restrict__ tile,
                                                   const int32_t* __restrict__ total,
                                                   int64_t* __restrict__ offsets,
                                                   int32_t* __restrict__ order,
                                                   int32_t* __restrict__ slot) {
  extern __shared__ int32_t next[];  // [PW][E]: pairs of each warp, then their next slots
  __shared__ int32_t part[PW];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int PER = PTILE / PW;
  const int64_t base = (int64_t)blockIdx.x * PTILE + warp * PER;
  int mine[PER / 32];  // the warp's pairs, 32 consecutive ones at a time; -1: none
#pragma unroll
  for (int j = 0; j < PER / 32; ++j) {
    const int64_t i = base + j * 32 + lane;
    mine[j] = i < pairs ? experts[i] : -1;
    if (mine[j] < 0 || mine[j] >= E) mine[j] = -1;
  }
  for (int e = tid; e < PW * E; e += PT) next[e] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER / 32; ++j)
    if (mine[j] >= 0) atomicAdd(&next[warp * E + mine[j]], 1);
  __syncthreads();
  // offsets: each thread takes MAX_E / PT consecutive experts at most
  constexpr int Q = MAX_E / PT;
  const int q = (E + PT - 1) / PT;
  int32_t count[Q], sum = 0;
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    const int e = tid * q + j;
    count[j] = 0;
    if (j < q && e < E) {
      if (tiles > 1)
        count[j] = total[e];
      else
        for (int w = 0; w < PW; ++w) count[j] += next[w * E + e];
    }
    sum += count[j];
  }
  int32_t to = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t y = __shfl_up_sync(0xffffffffu, to, o);
    if (lane >= o) to += y;
  }
  if (lane == 31) part[warp] = to;
  __syncthreads();
  int32_t at = to - sum, placed = 0;
#pragma unroll
  for (int w = 0; w < PW; ++w) {
    if (w < warp) at += part[w];
    placed += part[w];
  }
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    const int e = tid * q + j;
    if (j < q && e < E) {
      if (blockIdx.x == 0) offsets[e] = at;
      int32_t first = at + (tiles > 1 ? tile[(int64_t)e * tiles + blockIdx.x] : 0);
      for (int w = 0; w < PW; ++w) {
        const int32_t c = next[w * E + e];
        next[w * E + e] = first;
        first += c;
      }
    }
    at += count[j];
  }
  if (blockIdx.x == 0 && tid == 0) offsets[E] = placed;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER / 32; ++j) {  // in order
    const int64_t i = base + j * 32 + lane;
    const bool some = mine[j] >= 0;
    const unsigned same = __match_any_sync(0xffffffffu, some ? mine[j] : -1);
    int32_t p = -1;
    if (some) p = next[warp * E + mine[j]] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (some && lane == 31 - __clz(same)) next[warp * E + mine[j]] = p + 1;
    __syncwarp();
    if (some) order[p] = (int32_t)i;
    if (i < pairs) {
      slot[i] = p;
      if (i >= placed) order[i] = -1;
    }
  }
}

// ------------------------------------------------------------------------------------------------
// rows of vectors: B bytes (16 where every row starts on 16 bytes, down to one element) at a time
// ------------------------------------------------------------------------------------------------
template <int B>
struct Bytes;
template <>
struct Bytes<16> { using type = uint4; };
template <>
struct Bytes<8> { using type = uint2; };
template <>
struct Bytes<4> { using type = unsigned; };
template <>
struct Bytes<2> { using type = unsigned short; };

template <class T, int B>
union Piece {
  static constexpr int N = B / sizeof(T);
  typename Bytes<B>::type raw;
  T t[N];
  __device__ __forceinline__ Piece() {}
};

constexpr int XT = 256;  // threads of a block

// A thread takes a piece of a row, K of the row's pairs in flight and the next row's slots and
// weights on their way: the combined row is written once and every y row read once.  Bound by
// memory: 20,000 rows of 512 bf16, 4 experts each: 18.4 us, 5.6 TB/s.
template <class T, int B, int K>
__global__ void __launch_bounds__(XT) k_combine(int64_t rows, int k, int pieces, int wide,
                                                const T* __restrict__ y,
                                                const int32_t* __restrict__ slot,
                                                const float* __restrict__ weights,
                                                T* __restrict__ out) {
  using P = Piece<T, B>;
  using V = typename Bytes<B>::type;
  const int per = XT / wide, tr = threadIdx.x / wide, tc = threadIdx.x % wide;
  if (tr >= per) return;
  const unsigned pairs = (unsigned)(rows * k);
  const int64_t step = (int64_t)gridDim.x * per;
  int64_t t = (int64_t)blockIdx.x * per + tr;
  unsigned p[K], pn[K];  // a pair that is none has a slot of at least `pairs`
  float w[K], wn[K];
  auto fetch = [&](int64_t row, int j0, unsigned* q, float* f) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const bool in = row < rows && j0 + j < k;
      q[j] = in ? (unsigned)__ldg(slot + row * k + j0 + j) : 0xffffffffu;
      f[j] = in && weights ? __ldg(weights + row * k + j0 + j) : 1.f;
    }
  };
  fetch(t, 0, pn, wn);
  for (; t < rows; t += step) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      p[j] = pn[j];
      w[j] = wn[j];
    }
    fetch(t + step, 0, pn, wn);
    for (int c = tc; c < pieces; c += wide) {
      float s[P::N];
#pragma unroll
      for (int i = 0; i < P::N; ++i) s[i] = 0.f;
      for (int j0 = 0; j0 < k; j0 += K) {
        if (k > K) fetch(t, j0, p, w);
        P v[K];
#pragma unroll
        for (int j = 0; j < K; ++j)
          if (p[j] < pairs) v[j].raw = __ldcs(reinterpret_cast<const V*>(y) + (int64_t)p[j] * pieces + c);
#pragma unroll
        for (int j = 0; j < K; ++j)
          if (p[j] < pairs) {
#pragma unroll
            for (int i = 0; i < P::N; ++i) s[i] = fmaf(w[j], to_f32(v[j].t[i]), s[i]);
          }
      }
      P o;
#pragma unroll
      for (int i = 0; i < P::N; ++i) o.t[i] = from_f32<T>(s[i]);
      reinterpret_cast<V*>(out)[t * pieces + c] = o.raw;
    }
  }
}

template <class T, int B>
__device__ __forceinline__ void zero_rows(int64_t pairs, int pieces, const int64_t* placed, T* out) {
  using V = typename Bytes<B>::type;
  const int64_t from = *placed < 0 ? 0 : *placed;
  if (from >= pairs) return;
  Piece<T, B> z;
#pragma unroll
  for (int i = 0; i < Piece<T, B>::N; ++i) z.t[i] = from_f32<T>(0.f);
  const int64_t end = pairs * pieces;
  for (int64_t i = from * pieces + (int64_t)blockIdx.x * XT + threadIdx.x; i < end;
       i += (int64_t)gridDim.x * XT)
    reinterpret_cast<V*>(out)[i] = z.raw;
}

// xs[slot] = x[row]: a row is read once and written to each of its slots
template <class T, int B>
__global__ void __launch_bounds__(XT) k_gather(int64_t rows, int k, int pieces, int wide,
                                               const T* __restrict__ x,
                                               const int32_t* __restrict__ slot,
                                               const int64_t* __restrict__ placed,
                                               T* __restrict__ xs) {
  using V = typename Bytes<B>::type;
  const int per = XT / wide, tr = threadIdx.x / wide, tc = threadIdx.x % wide;
  const int64_t pairs = rows * k;
  if (tr < per)
    for (int64_t t = (int64_t)blockIdx.x * per + tr; t < rows; t += (int64_t)gridDim.x * per)
      for (int c = tc; c < pieces; c += wide) {
        const V v = __ldg(reinterpret_cast<const V*>(x) + t * pieces + c);
        for (int j = 0; j < k; ++j) {
          const int32_t p = __ldg(slot + t * k + j);
          if (p >= 0 && p < pairs) reinterpret_cast<V*>(xs)[(int64_t)p * pieces + c] = v;
        }
      }
  zero_rows<T, B>(pairs, pieces, placed, xs);
}

// dy[slot] = weight dout[row] and dweights = dout[row] . y[slot]: a warp takes a row, KG of its pairs
// at a time, so dout is read once (from L1 for more pairs) and each y row is read where its dy row is
// written.  Bound by memory: 32,768 rows of 1024 bf16, 8 experts each: 177 us, 6.5 TB/s.
template <class T, int B, int KG>
__global__ void __launch_bounds__(XT) k_combine_backward(
    int64_t rows, int k, int pieces, const T* __restrict__ dout, const T* __restrict__ y,
    const int32_t* __restrict__ slot, const int64_t* __restrict__ placed,
    const float* __restrict__ weights, T* __restrict__ dy, float* __restrict__ dweights) {
  using P = Piece<T, B>;
  using V = typename Bytes<B>::type;
  const int lane = threadIdx.x & 31;
  const int64_t pairs = rows * k;
  for (int64_t t = ((int64_t)blockIdx.x * XT + threadIdx.x) >> 5; t < rows;
       t += (int64_t)gridDim.x * (XT / 32))
    for (int j0 = 0; j0 < k; j0 += KG) {
      int64_t at[KG];
      float w[KG], s[KG];
#pragma unroll
      for (int j = 0; j < KG; ++j) {
        const int32_t p = j0 + j < k ? __ldg(slot + t * k + j0 + j) : -1;
        at[j] = p >= 0 && p < pairs ? (int64_t)p * pieces : -1;
        w[j] = at[j] >= 0 ? __ldg(weights + t * k + j0 + j) : 0.f;
        s[j] = 0.f;
      }
      for (int c = lane; c < pieces; c += 32) {
        P g, v[KG];
        g.raw = __ldg(reinterpret_cast<const V*>(dout) + t * pieces + c);
#pragma unroll
        for (int j = 0; j < KG; ++j)
          if (at[j] >= 0) v[j].raw = __ldg(reinterpret_cast<const V*>(y) + at[j] + c);
#pragma unroll
        for (int j = 0; j < KG; ++j)
          if (at[j] >= 0) {
            P o;
#pragma unroll
            for (int i = 0; i < P::N; ++i) {
              const float f = to_f32(g.t[i]);
              s[j] = fmaf(f, to_f32(v[j].t[i]), s[j]);
              o.t[i] = from_f32<T>(w[j] * f);
            }
            reinterpret_cast<V*>(dy)[at[j] + c] = o.raw;
          }
      }
#pragma unroll
      for (int j = 0; j < KG; ++j) {
#pragma unroll
        for (int o = 16; o; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
        if (lane == 0 && j0 + j < k) dweights[t * k + j0 + j] = s[j];
      }
    }
  zero_rows<T, B>(pairs, pieces, placed, dy);
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
// blocks for `work` units of a block each, at most so many an SM
unsigned grid_of(int64_t work, int blocks_an_sm) {
  const int64_t most = (int64_t)blocks_an_sm * sm_count();
  return (unsigned)(work < most ? (work > 0 ? work : 1) : most);
}
// threads that share a row of `pieces`: whole warps, or a power of two below one
int threads_wide(int64_t pieces) {
  if (pieces >= XT) return XT;
  if (pieces > 32) return (int)((pieces + 31) / 32 * 32);
  int w = 1;
  while (w < pieces) w *= 2;
  return w;
}
// calls f(B) for the largest piece of at most 16 bytes that divides a row and every base address
template <class T, class F>
erc_status with_bytes(int64_t width, std::initializer_list<const void*> bases, F&& f) {
  uintptr_t all = (uintptr_t)(width * sizeof(T));
  for (const void* p : bases) all |= reinterpret_cast<uintptr_t>(p);
  if (all % 16 == 0) return f(std::integral_constant<int, 16>());
  if (all % 8 == 0) return f(std::integral_constant<int, 8>());
  if constexpr (sizeof(T) == 2) {
    if (all % 4 != 0) return f(std::integral_constant<int, 2>());
  }
  return f(std::integral_constant<int, 4>());
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" size_t erc_expert_plan_workspace_size(int64_t rows, int32_t k, int32_t experts) {
  if (rows < 0 || k < 1 || k > ERC_ROUTE_MAX_K || rows > 0x7fffffffLL / k || experts < 1 ||
      experts > MAX_E)
    return 0;
  if (plan_tiles(rows * k) <= 1) return 0;  // a single block plans them
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
  const int64_t tiles = plan_tiles(pairs);
  if (tiles > 1 && (!ws || ws_bytes < erc_expert_plan_workspace_size(rows, k, n_experts)))
    return set_error(ERC_ERR_CAPACITY, "workspace too small");
  Plan p = {};
  if (tiles > 1) {
    Arena ar(reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~uintptr_t(255)));
    plan_experts(ar, p, pairs, n_experts);
    k_plan_count<<<(unsigned)tiles, PT, 0, s>>>(experts, pairs, n_experts, (int)tiles, p.tile);
    k_plan_scan<<<n_experts, PT, 0, s>>>(p.tile, (int)tiles, p.total);
    count_launches(2);
  }
  k_plan_place<<<(unsigned)tiles, PT, PW * n_experts * sizeof(int32_t), s>>>(
      experts, pairs, n_experts, (int)tiles, p.tile, p.total, offsets, order, slot);
  count_launches(1);
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
    return with_bytes<T>(width, {y, out}, [&](auto bytes) {
      constexpr int B = decltype(bytes)::value;
      const int pieces = (int)(width * sizeof(T) / B), wide = threads_wide(pieces);
      const unsigned grid = grid_of((rows + XT / wide - 1) / (XT / wide), 4);
      auto kernel = k <= 2 ? k_combine<T, B, 2> : k <= 4 ? k_combine<T, B, 4> : k_combine<T, B, 8>;
      kernel<<<grid, XT, 0, as_stream(stream)>>>(rows, k, pieces, wide, static_cast<const T*>(y), slot,
                                                 weights, static_cast<T*>(out));
      count_launches(1);
      ERC_CUDA(cudaGetLastError());
      return ERC_OK;
    });
  });
}

extern "C" erc_status erc_expert_gather(int64_t rows, int32_t k, int64_t width, const void* x,
                                        int32_t type, const int32_t* slot, const int64_t* placed,
                                        void* xs, erc_stream stream) {
  clear_error();
  ERC_TRY(check_sizes(rows, k, width, type));
  if (rows == 0 || width == 0) return ERC_OK;
  ERC_REQUIRE(x && slot && placed && xs, "null pointer");
  ERC_REQUIRE(aligned(x, type) && aligned(xs, type), "misaligned x or xs");
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    return with_bytes<T>(width, {x, xs}, [&](auto bytes) {
      constexpr int B = decltype(bytes)::value;
      const int pieces = (int)(width * sizeof(T) / B), wide = threads_wide(pieces);
      const unsigned grid = grid_of((rows + XT / wide - 1) / (XT / wide), 32);
      k_gather<T, B><<<grid, XT, 0, as_stream(stream)>>>(rows, k, pieces, wide,
                                                         static_cast<const T*>(x), slot, placed,
                                                         static_cast<T*>(xs));
      count_launches(1);
      ERC_CUDA(cudaGetLastError());
      return ERC_OK;
    });
  });
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
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    return with_bytes<T>(width, {dout, y, dy}, [&](auto bytes) {
      constexpr int B = decltype(bytes)::value;
      const int pieces = (int)(width * sizeof(T) / B);
      auto kernel = k == 1   ? k_combine_backward<T, B, 1>
                    : k <= 2 ? k_combine_backward<T, B, 2>
                             : k_combine_backward<T, B, 4>;
      kernel<<<grid_of((rows + XT / 32 - 1) / (XT / 32), 32), XT, 0, as_stream(stream)>>>(
          rows, k, pieces, static_cast<const T*>(dout), static_cast<const T*>(y), slot, placed, weights,
          static_cast<T*>(dy), dweights);
      count_launches(1);
      ERC_CUDA(cudaGetLastError());
      return ERC_OK;
    });
  });
}
