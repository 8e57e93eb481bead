// route.cu -- experts of a row from its scores, and the gradient of the chosen weights.
//
// s = softmax(l) or 1 / (1 + exp(-l)) with choice.cuh's exponential: the softmax normaliser is a sum
// of integer weights, every other step one rounded float32 operation, so the choice s + bias and
// with it the chosen experts have the same bits on every machine.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int QW = 4;  // rows (one warp each) of a block
constexpr int MAX_E = ERC_ROUTE_MAX_EXPERTS;

// scores of one row into sc[] (shared, the warp's own); masked entries get -1
template <class T>
__device__ __forceinline__ void row_scores(const T* x, int E, int score, float* sc, int lane) {
  if (score == ERC_SCORE_SIGMOID) {
    for (int i = lane; i < E; i += 32) {
      const float l = clean_score(to_f32(x[i]));
      const float e = pow2_float(-__fmul_rn(fabsf(l), LOG2E), -126.f);
      sc[i] = l == -INFINITY ? -1.f : __fdiv_rn(l >= 0.f ? 1.f : e, __fadd_rn(1.f, e));
    }
  } else {
    unsigned k = 0;
    for (int i = lane; i < E; i += 32) k = max(k, order_key(clean_score(to_f32(x[i]))));
    const float m = order_value(__reduce_max_sync(0xffffffffu, k));
    unsigned long long z = 0;
    for (int i = lane; i < E; i += 32) {
      const float l = clean_score(to_f32(x[i]));
      if (l != -INFINITY) z += fixed_weight(below_max(l, m, LOG2E));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    const float inv = __frcp_rn(__fmul_rn(__ull2float_rn(z ? z : 1ull), 9.094947017729282e-13f));
    for (int i = lane; i < E; i += 32) {
      const float l = clean_score(to_f32(x[i]));
      sc[i] = l == -INFINITY ? -1.f : __fmul_rn(pow2_float(below_max(l, m, LOG2E), -41.f), inv);
    }
  }
  __syncwarp();
}

// (largest key, lowest index) over the warp
__device__ __forceinline__ void warp_best(unsigned& key, int& index) {
  const unsigned best = __reduce_max_sync(0xffffffffu, key);
  const unsigned i = __reduce_min_sync(0xffffffffu, key == best ? (unsigned)index : 0xffffffffu);
  key = best;
  index = (int)i;
}

template <class T>
__global__ void __launch_bounds__(QW * 32) k_route(int64_t rows, const T* __restrict__ logits,
                                                   int64_t stride, const float* __restrict__ bias,
                                                   erc_route_rule rule, int32_t* __restrict__ experts,
                                                   float* __restrict__ weights) {
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = rule.experts, k = rule.k, G = rule.groups;
  const int64_t row = (int64_t)blockIdx.x * QW + warp;
  if (row >= rows) return;
  float* sc = smem + warp * (2 * E + G);
  unsigned* key = reinterpret_cast<unsigned*>(sc + E);  // 0: not to be chosen
  unsigned* gkey = key + E;
  row_scores(logits + row * stride, E, rule.score, sc, lane);
  for (int i = lane; i < E; i += 32) {
    const float c = bias ? __fadd_rn(sc[i], bias[i]) : sc[i];
    key[i] = sc[i] < 0.f || c != c || c == -INFINITY ? 0u : order_key(__fadd_rn(c, 0.f));
  }
  __syncwarp();
  if (G > 1 && rule.top_groups < G) {
    const int size = E / G;
    for (int g = lane; g < G; g += 32) {
      unsigned a = 0, b = 0;
      for (int i = g * size; i < (g + 1) * size; ++i) {
        const unsigned v = key[i];
        b = max(b, min(a, v));
        a = max(a, v);
      }
      float s = a ? order_value(a) : -INFINITY;
      if (b && rule.group_best == 2) s = __fadd_rn(s, order_value(b));
      gkey[g] = a ? order_key(__fadd_rn(s, 0.f)) : 0u;
    }
    __syncwarp();
    // mark the best groups: a marked group's key becomes 1, a passed-over one's members 0
    for (int t = 0; t < rule.top_groups; ++t) {
      unsigned b = 0;
      int bi = 0x7fffffff;
      for (int g = lane; g < G; g += 32)
        if (gkey[g] > b && gkey[g] != 1u) { b = gkey[g]; bi = g; }
      warp_best(b, bi);
      if (b == 0) break;
      if (lane == 0) gkey[bi] = 1u;
      __syncwarp();
    }
    for (int i = lane; i < E; i += 32)
      if (gkey[i / size] != 1u) key[i] = 0u;
    __syncwarp();
  }
  float sum = 0.f, mine = 0.f;
  int chosen = -1;
  for (int j = 0; j < k; ++j) {
    unsigned b = 0;
    int bi = 0x7fffffff;
    for (int i = lane; i < E; i += 32)
      if (key[i] > b) { b = key[i]; bi = i; }
    warp_best(b, bi);
    const float s = b ? sc[bi] : 0.f;
    sum = __fadd_rn(sum, s);
    if (lane == j) {
      chosen = b ? bi : -1;
      mine = s;
    }
    __syncwarp();
    if (b && lane == 0) key[bi] = 0u;
    __syncwarp();
  }
  if (lane < k) {
    if (rule.renorm) mine = sum > 0.f ? __fdiv_rn(mine, sum) : 0.f;
    experts[row * k + lane] = chosen;
    weights[row * k + lane] = __fmul_rn(mine, rule.scale);
  }
}

template <class T>
__global__ void __launch_bounds__(QW * 32)
    k_route_backward(int64_t rows, const T* __restrict__ logits, int64_t stride,
                     const int32_t* __restrict__ experts, const float* __restrict__ dweights,
                     erc_route_rule rule, T* __restrict__ dlogits) {
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = rule.experts, k = rule.k;
  const int64_t row = (int64_t)blockIdx.x * QW + warp;
  if (row >= rows) return;
  float* sc = smem + warp * 2 * E;
  float* ds = sc + E;
  row_scores(logits + row * stride, E, rule.score, sc, lane);
  for (int i = lane; i < E; i += 32) ds[i] = 0.f;
  __syncwarp();
  const int at = lane < k ? experts[row * k + lane] : -1;
  const bool some = at >= 0 && at < E;
  const float s = some ? fmaxf(sc[at], 0.f) : 0.f;
  float g = some ? dweights[row * k + lane] * rule.scale : 0.f;
  auto sum = [](float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  if (rule.renorm) {
    const float D = sum(s);
    const float p = D > 0.f ? s / D : 0.f;
    const float gp = sum(g * p);
    g = some && D > 0.f ? (g - gp) / D : 0.f;
  }
  const float gs = sum(g * s);
  if (some) atomicAdd(&ds[at], g);
  __syncwarp();
  for (int i = lane; i < E; i += 32) {
    const float v = fmaxf(sc[i], 0.f);
    const float d = rule.score == ERC_SCORE_SIGMOID ? ds[i] * v * (1.f - v) : v * (ds[i] - gs);
    dlogits[row * E + i] = from_f32<T>(d);
  }
}

erc_status check_rule(const erc_route_rule* r, int32_t type, int64_t rows, int64_t stride) {
  ERC_REQUIRE(r, "rule is required");
  ERC_REQUIRE(type >= ERC_F32 && type <= ERC_F16, "bad score type %d", type);
  ERC_REQUIRE(rows >= 0 && rows <= 0x7fffffffLL, "rows must be in [0, 2^31)");
  ERC_REQUIRE(r->experts >= 1 && r->experts <= MAX_E, "experts must be in [1, %d]", MAX_E);
  ERC_REQUIRE(r->k >= 1 && r->k <= ERC_ROUTE_MAX_K && r->k <= r->experts,
              "k must be in [1, min(%d, experts)]", ERC_ROUTE_MAX_K);
  ERC_REQUIRE(r->score == ERC_SCORE_SOFTMAX || r->score == ERC_SCORE_SIGMOID, "bad score kind %d",
              r->score);
  ERC_REQUIRE(r->groups >= 1 && r->experts % r->groups == 0, "groups must divide experts");
  ERC_REQUIRE(r->top_groups >= 1 && r->top_groups <= r->groups, "top_groups must be in [1, groups]");
  ERC_REQUIRE(r->group_best == 1 || r->group_best == 2, "group_best must be 1 or 2");
  ERC_REQUIRE(r->scale > -3.4e38f && r->scale < 3.4e38f, "scale must be finite");
  ERC_REQUIRE(stride >= 0, "stride must be >= 0");
  return ERC_OK;
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" erc_status erc_route(int64_t rows, const void* logits, int32_t type, int64_t stride,
                                const float* bias, const erc_route_rule* rule, int32_t* experts,
                                float* weights, erc_stream stream) {
  clear_error();
  ERC_TRY(check_rule(rule, type, rows, stride));
  if (rows == 0) return ERC_OK;
  ERC_REQUIRE(logits && experts && weights, "null pointer");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(logits) % type_bytes(type) == 0, "misaligned logits");
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const size_t sh = QW * (2 * rule->experts + rule->groups) * sizeof(float);
    k_route<T><<<(unsigned)((rows + QW - 1) / QW), QW * 32, sh, as_stream(stream)>>>(
        rows, static_cast<const T*>(logits), stride, bias, *rule, experts, weights);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}

extern "C" erc_status erc_route_backward(int64_t rows, const void* logits, int32_t type,
                                         int64_t stride, const int32_t* experts,
                                         const float* dweights, const erc_route_rule* rule,
                                         void* dlogits, erc_stream stream) {
  clear_error();
  ERC_TRY(check_rule(rule, type, rows, stride));
  if (rows == 0) return ERC_OK;
  ERC_REQUIRE(logits && experts && dweights && dlogits, "null pointer");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(logits) % type_bytes(type) == 0 &&
                  reinterpret_cast<uintptr_t>(dlogits) % type_bytes(type) == 0,
              "misaligned logits or dlogits");
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const size_t sh = QW * 2 * rule->experts * sizeof(float);
    k_route_backward<T><<<(unsigned)((rows + QW - 1) / QW), QW * 32, sh, as_stream(stream)>>>(
        rows, static_cast<const T*>(logits), stride, experts, dweights, *rule,
        static_cast<T*>(dlogits));
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
