// route.cu -- experts of a row from its scores, and the gradient of the chosen weights.
//
// s = softmax(l) or 1 / (1 + exp(-l)) with choice.cuh's exponential: the softmax normaliser is a sum
// of integer weights, every other step one rounded float32 operation, so the choice s + bias and
// with it the chosen experts have the same bits on every machine.  2^t is kept down to rint(t) = -126, so
// that experts far below the best keep their order and their weights; only the integers end at 2^-41.
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
      sc[i] = l == -INFINITY ? -1.f : __fmul_rn(pow2_float(below_max(l, m, LOG2E), -126.f), inv);
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

// ------------------------------------------------------------------------------------------------
// rows in registers: L lanes take a row, each V consecutive experts, so a warp takes 32 / L rows and
// the lowest index among equals is the lowest (lane, place).
// ------------------------------------------------------------------------------------------------
constexpr int FW = 8;  // warps of a block

template <int L>
__device__ __forceinline__ unsigned lanes_max(unsigned v) {
  if constexpr (L == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}
template <int L>
__device__ __forceinline__ unsigned lanes_sum(unsigned v) {
  if constexpr (L == 32) {
    return __reduce_add_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// V scores of a lane from `first` on; masked from E on.  `wide`: 16-byte loads are aligned and V
// divides E.
template <class T, int V>
__device__ __forceinline__ void load_scores(const T* x, int first, int E, bool wide, bool row,
                                            float* l) {
  constexpr int N = ScoreVec<T>::N;
  if (!row || first >= E) {
#pragma unroll
    for (int j = 0; j < V; ++j) l[j] = -INFINITY;
  } else if (wide) {
#pragma unroll
    for (int j = 0; j < V / N; ++j)
      unpack_scores(__ldg(reinterpret_cast<const uint4*>(x + first) + j), l + j * N, T());
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      l[j] = first + j < E ? fmaxf(to_f32(x[first + j]), -INFINITY) : -INFINITY;
  }
}

struct RowScale {  // of a softmax row: its maximum and 1 / Z
  float max, inv;
};

// one logit's score, -1 where masked
template <bool SIGMOID>
__device__ __forceinline__ float one_score(float l, const RowScale& r) {
  if (l == -INFINITY) return -1.f;
  if (!SIGMOID) return __fmul_rn(pow2_float(below_max(l, r.max, LOG2E), -126.f), r.inv);
  const float e = pow2_float(-__fmul_rn(fabsf(l), LOG2E), -126.f);
  return __fdiv_rn(l >= 0.f ? 1.f : e, __fadd_rn(1.f, e));
}

// 2^k for the sum k + 1.5 2^23 that pow2_pair gives, k in [-126, 0].  A product with it may be subnormal
// (k = -126), which adding k to the other factor's exponent bits could not give.
__device__ __forceinline__ float two_to(float k_shifted) {
  return __uint_as_float((__float_as_uint(k_shifted) << 23) + 0x3f800000u);
}

// the scores s_j of a lane's logits, -1 where masked
template <int L, int V, bool SIGMOID>
__device__ __forceinline__ RowScale lane_scores(const float* l, float* s) {
  RowScale r = {};
  if (SIGMOID) {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      float t[2], p[2], k[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) t[i] = fmaxf(-__fmul_rn(fabsf(l[j + i]), LOG2E), -200.f);
      pow2_pair(t[0], t[1], p, k);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x = l[j + i];
        const float e = t[i] >= -126.5f ? __fmul_rn(p[i], two_to(k[i])) : 0.f;
        s[j + i] = x == -INFINITY ? -1.f : __fdiv_rn(x >= 0.f ? 1.f : e, __fadd_rn(1.f, e));
      }
    }
  } else {
    float m = l[0];
#pragma unroll
    for (int j = 1; j < V; ++j) m = fmaxf(m, l[j]);
    m = order_value(lanes_max<L>(order_key(__fadd_rn(m, 0.f))));
    unsigned hi = 0, lo = 0;
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      float t[2], p[2], k[2];
      unsigned h[2], w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        t[i] = l[j + i] == -INFINITY ? -200.f : fmaxf(below_max(l[j + i], m, LOG2E), -200.f);
      pow2_pair(t[0], t[1], p, k);
#pragma unroll
      for (int i = 0; i < 2; ++i) s[j + i] = t[i] >= -126.5f ? __fmul_rn(p[i], two_to(k[i])) : 0.f;
      split_weights(pair(s[j], s[j + 1]), h, w);
      hi += h[0] + h[1];
      lo += w[0] + w[1];
    }
    hi = lanes_sum<L>(hi - V * BIAS);
    lo = lanes_sum<L>(lo - V * BIAS);
    const unsigned long long z = ((unsigned long long)hi << 20) + lo;
    const float inv = __frcp_rn(__fmul_rn(__ull2float_rn(z ? z : 1ull), 9.094947017729282e-13f));
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = l[j] == -INFINITY ? -1.f : __fmul_rn(s[j], inv);
    r.max = m;
    r.inv = inv;
  }
  return r;
}

// the choice of an expert from its score (negative: masked): -inf where it is not to be chosen.  A score
// is never -0, so neither is its sum with a bias.
__device__ __forceinline__ float choice(float s, float bias) {
  return s < 0.f ? -INFINITY : fmaxf(__fadd_rn(s, bias), -INFINITY);
}
template <int V>
__device__ __forceinline__ void lane_bias(const float* bias, int first, int E, float* b) {
#pragma unroll
  for (int j = 0; j < V; ++j) b[j] = bias && first + j < E ? __ldg(bias + first + j) : 0.f;
}

template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  if constexpr (L == 32) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
  } else {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}

// the score of a lane's group (a power of two of lanes): its best choice, or the sum of its best two;
// `terms`: the sum of their magnitudes, -1 where there is no choice
template <int V>
__device__ __forceinline__ float group_score(const erc_route_rule& rule, int span, const float* c,
                                             float& terms) {
  float a = -INFINITY, b = -INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    b = fmaxf(b, fminf(a, c[j]));
    a = fmaxf(a, c[j]);
  }
  for (int o = 1; o < span; o <<= 1) {
    const float a2 = __shfl_xor_sync(0xffffffffu, a, o), b2 = __shfl_xor_sync(0xffffffffu, b, o);
    b = fmaxf(fmaxf(b, b2), fminf(a, a2));
    a = fmaxf(a, a2);
  }
  const bool two = b > -INFINITY && rule.group_best == 2;
  terms = two ? fabsf(a) + fabsf(b) : a > -INFINITY ? fabsf(a) : -1.f;
  return two ? __fadd_rn(a, b) : a;
}

// The choices of the groups passed over become -inf; ties go to the lowest group.  Scores are compared
// as keys, with 0 for a group with no choice: a sum of two may be -inf, and that is still above none.
template <int L, int V>
__device__ __forceinline__ void keep_groups(const erc_route_rule& rule, int lane, float* c) {
  const int at = lane % L, span = rule.experts / rule.groups / V;
  float terms;
  const float score = group_score<V>(rule, span, c, terms);
  const unsigned mine = terms < 0.f ? 0u : order_key(score);
  int better = 0;
  for (int o = 0; o < rule.groups; ++o) {
    const unsigned other = __shfl_sync(0xffffffffu, mine, lane - at + o * span);
    better += other > mine || (other == mine && o < at / span);
  }
  if (better >= rule.top_groups) {
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = -INFINITY;
  }
}

// k rounds over a row of L lanes: the best choice, by its first owner, is taken away
template <int L, int V>
__device__ __forceinline__ void pick_in_rounds(const erc_route_rule& rule, int lane, bool live,
                                               int64_t row, const float* s, float* c, float* picked,
                                               int32_t* experts, float* weights) {
  const int at = lane % L, k = rule.k;
  const unsigned mates = (L == 32 ? 0xffffffffu : ((1u << (L & 31)) - 1)) << (lane - at);
  float sum = 0.f, top = -INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j) top = fmaxf(top, c[j]);
  for (int i = 0; i < k; ++i) {
    const float best = lanes_max<L>(top);
    const int owner = __ffs(__ballot_sync(0xffffffffu, top == best) & mates) - 1;
    const bool take = lane == owner && best > -INFINITY;
    int place = V;
    float score = 0.f;
    top = -INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (take && c[j] == best && place == V) {
        place = j;
        score = s[j];
        c[j] = -INFINITY;
      }
      top = fmaxf(top, c[j]);
    }
    score = __shfl_sync(0xffffffffu, score, owner);
    sum = __fadd_rn(sum, score);
    if (lane == owner && live) {
      picked[i] = score;
      experts[row * k + i] = take ? at * V + place : -1;
    }
  }
  __syncwarp();
  for (int i = at; i < k && live; i += L) {
    float w = picked[i];
    if (rule.renorm) w = sum > 0.f ? __fdiv_rn(w, sum) : 0.f;
    weights[row * k + i] = __fmul_rn(w, rule.scale);
  }
  __syncwarp();
}

// rows of at most 128 experts: L = 8 or 16 lanes a row
template <class T, int L, int V, bool SIGMOID>
__global__ void __launch_bounds__(FW * 32)
    k_route_lanes(int64_t rows, const T* __restrict__ logits, int64_t stride,
                  const float* __restrict__ bias, erc_route_rule rule, bool wide,
                  int32_t* __restrict__ experts, float* __restrict__ weights) {
  constexpr int R = 32 / L;  // rows of a warp
  __shared__ float picked[FW * R][ERC_ROUTE_MAX_K];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / L;
  const int E = rule.experts, first = lane % L * V;
  const int64_t row = ((int64_t)blockIdx.x * FW + warp) * R + sub;
  const bool live = row < rows;
  float l[V], s[V], c[V];
  load_scores<T, V>(logits + (live ? row : 0) * stride, first, E, wide, live, l);
  lane_scores<L, V, SIGMOID>(l, s);
  lane_bias<V>(bias, first, E, c);
#pragma unroll
  for (int j = 0; j < V; ++j) c[j] = choice(s[j], c[j]);
  if (rule.groups > 1 && rule.top_groups < rule.groups) keep_groups<L, V>(rule, lane, c);
  pick_in_rounds<L, V>(rule, lane, live, row, s, c, picked[warp * R + sub], experts, weights);
}

// The places of the choices that can be among the k best into `list`, in ascending order: those no
// lower than the k-th distinct best of the lanes' best, less `margin` times (1 + its value).  Returns
// their number; more than 32 are not listed.
template <int V>
__device__ __forceinline__ int candidates(const float* c, int k, int first, float margin,
                                          uint16_t* list) {
  float top = -INFINITY, theta = -INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j) top = fmaxf(top, c[j]);
  for (int i = 0; i < k; ++i) {
    theta = lanes_max<32>(top);
    if (theta == -INFINITY) break;
    if (top == theta) top = -INFINITY;
  }
  const float least = margin > 0.f && theta > -INFINITY ? theta - margin * (1.f + fabsf(theta)) : theta;
  if (least != least) return 33;  // a choice of +inf has no margin
  unsigned mask = 0;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (c[j] >= least && c[j] > -INFINITY) mask |= 1u << j;
  int to = __popc(mask);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, to, o);
    if ((int)(threadIdx.x & 31) >= o) to += y;
  }
  const int n = __shfl_sync(0xffffffffu, to, 31);
  if (n > 32) return n;
  for (to -= __popc(mask); mask; mask &= mask - 1) list[to++] = (uint16_t)(first + __ffs(mask) - 1);
  __syncwarp();
  return n;
}

// Rows of more than 128 experts: a warp a row, the k best ranked among at most 32 candidates, one a
// lane, by their exact choices.  For sigmoid scores the candidates come from the hardware's
// exponential and reciprocal: with |t| as computed here their scores are within 1.1e-6 of the exact
// ones (2^-22 for ex2, 1.9e-7 for the polynomial, an ulp for rcp, three roundings), so 4e-6 (1 + |c|)
// covers twice that and the rounding of the sum with the bias (2^-23 |c| between two choices).  A group's
// score adds two such errors and its own rounding, all in proportion to its terms, which may be far
// larger than their sum: 2.2e-6 + 2.4e-7 (|a| + |b|), and for two groups less than 8e-6 (1 + the largest
// |a| + |b| of the row).  Rows whose groups are not told apart by that, or with more candidates, take
// exact choices and, if need be, k rounds.
//
// A warp takes rows in turn, its biases in registers and the next row on its way.
//
// E = 256, k = 8, four of eight groups, sigmoid with bias, 32,768 rows of bf16: 32 us, 761 instructions a
// row, issued in 0.60 of the cycles; k rounds over exact scores took 55 us (1505 instructions).
template <class T, int V, bool SIGMOID>
__global__ void __launch_bounds__(FW * 32, V == 8 ? 4 : V == 16 ? 2 : 1)
    k_route_warp(int64_t rows, const T* __restrict__ logits, int64_t stride,
                 const float* __restrict__ bias, erc_route_rule rule, bool wide,
                 int32_t* __restrict__ experts, float* __restrict__ weights) {
  __shared__ float picked[FW][ERC_ROUTE_MAX_K];
  __shared__ uint16_t lists[FW][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = rule.experts, k = rule.k, first = lane * V;
  const bool grouped = rule.groups > 1 && rule.top_groups < rule.groups;
  const int span = grouped ? E / rule.groups / V : 32;
  const int64_t step = (int64_t)gridDim.x * FW;
  float b[V], next[V];
  lane_bias<V>(bias, first, E, b);
  int64_t row = (int64_t)blockIdx.x * FW + warp;
  load_scores<T, V>(logits + row * stride, first, E, wide, row < rows, next);
  for (; row < rows; row += step) {
    const T* x = logits + row * stride;
    float l[V], s[V], c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) l[j] = next[j];
    if (row + step < rows) load_scores<T, V>(x + step * stride, first, E, wide, true, next);
    int n = 33;
    RowScale scale = {};
    if (SIGMOID) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float e, r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-__fmul_rn(fabsf(l[j]), LOG2E)));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
        c[j] = fmaxf((l[j] >= 0.f ? r : e * r) + b[j], -INFINITY);
        if (l[j] == -INFINITY) c[j] = -INFINITY;
      }
      bool clear = true;
      if (grouped) {
        // the top_groups distinct best groups' scores, and the best of the rest
        float terms, worst = -INFINITY;
        const float mine = group_score<V>(rule, span, c, terms);
        float rest = mine;
        terms = lanes_max<32>(terms);
        for (int i = 0; i < rule.top_groups; ++i) {
          worst = lanes_max<32>(rest);
          if (rest == worst) rest = -INFINITY;
        }
        rest = lanes_max<32>(rest);
        const int in = __popc(__ballot_sync(0xffffffffu, mine >= worst && first < E));
        clear = in == rule.top_groups * span && worst - rest > 8e-6f * (1.f + terms);
        if (mine < worst) {
#pragma unroll
          for (int j = 0; j < V; ++j) c[j] = -INFINITY;
        }
      }
      if (clear) n = candidates<V>(c, k, first, 4e-6f, lists[warp]);
    }
    if (n > 32) {
      scale = lane_scores<32, V, SIGMOID>(l, s);
#pragma unroll
      for (int j = 0; j < V; ++j) c[j] = choice(s[j], b[j]);
      if (grouped) keep_groups<32, V>(rule, lane, c);
      n = candidates<V>(c, k, first, 0.f, lists[warp]);
      if (n > 32) {
        pick_in_rounds<32, V>(rule, lane, true, row, s, c, picked[warp], experts, weights);
        continue;
      }
    }
    // one candidate a lane, in ascending order of experts
    int e = -1;
    float score = 0.f, mine = -INFINITY;
    if (lane < n) {
      e = lists[warp][lane];
      score = one_score<SIGMOID>(fmaxf(to_f32(x[e]), -INFINITY), scale);
      mine = choice(score, bias ? __ldg(bias + e) : 0.f);
    }
    int rank = 0;
    for (int i = 0; i < n; ++i) {
      const float other = __shfl_sync(0xffffffffu, mine, i);
      rank += i < lane ? other >= mine : other > mine;
    }
    const bool in = lane < n && rank < k;
    const float sum = rule.renorm ? lanes_sum<32>(in ? score : 0.f) : 0.f;
    if (in) {
      if (rule.renorm) score = sum > 0.f ? __fdiv_rn(score, sum) : 0.f;
      experts[row * k + rank] = e;
      weights[row * k + rank] = __fmul_rn(score, rule.scale);
    }
    if (lane >= n && lane < k) {  // fewer than k can be chosen
      experts[row * k + lane] = -1;
      weights[row * k + lane] = 0.f;
    }
    __syncwarp();
  }
}

// The gradient of the row's weights.  Where nothing is chosen it is -s_i gs for softmax, with
// gs = sum ds s (0 in exact arithmetic when renormalised), and 0 for sigmoid, whose rows are then not
// read at all; the lanes that hold a chosen expert's gradient store it over that.  The chosen experts'
// 2^t is the forward pass's; the others', and Z, take the hardware's exponential (2^-22 of itself) and
// float32 sums.  169,343 x 64 f32: relative error 1.9e-7 against 64 bits, 1.2e-7 for plain float32 steps.
//
// 169,343 rows of 64 f32, two experts each, softmax: 22.5 us, 4.0 TB/s; the chain of a row (choices,
// scores, two reductions) is what is left.
template <class T, int L, int V, bool SIGMOID>
__global__ void __launch_bounds__(FW * 32)
    k_route_lanes_backward(int64_t rows, const T* __restrict__ logits, int64_t stride,
                           const int32_t* __restrict__ experts, const float* __restrict__ dweights,
                           erc_route_rule rule, bool wide, bool wide_out, T* __restrict__ dlogits) {
  constexpr int R = 32 / L, N = ScoreVec<T>::N, KL = (ERC_ROUTE_MAX_K + L - 1) / L;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / L, at = lane % L;
  const int E = rule.experts, k = rule.k;
  const int64_t row = ((int64_t)blockIdx.x * FW + warp) * R + sub;
  const bool live = row < rows;
  const T* x = logits + (live ? row : 0) * stride;
  const int first = at * V;
  auto power = [](float t) {  // 2^t, 0 below 2^-126
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    return e;
  };
  // the row's choices, one or more a lane: their loads start before the row's
  int place[KL];
  float s[KL], g[KL], chosen[KL], share[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    const int c = at + i * L;
    place[i] = c < k && live ? __ldg(experts + row * k + c) : -1;
    g[i] = c < k && live ? __ldg(dweights + row * k + c) * rule.scale : 0.f;
  }
  float v[V], m = 0.f, inv = 0.f;
  if (!SIGMOID) load_scores<T, V>(x, first, E, wide, live, v);
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    if (place[i] < 0 || place[i] >= E) {
      place[i] = -1;
      g[i] = 0.f;
    }
    chosen[i] = place[i] >= 0 ? clean_score(to_f32(x[place[i]])) : -INFINITY;
  }
  if (!SIGMOID) {
    m = v[0];
#pragma unroll
    for (int j = 1; j < V; ++j) m = fmaxf(m, v[j]);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      v[j] = v[j] == -INFINITY ? 0.f : power(below_max(v[j], m, LOG2E));
      z += v[j];
    }
    z = lanes_sum<L>(z);
    inv = z > 0.f ? __frcp_rn(z) : 0.f;
  }
  float D = 0.f;
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    const float l = chosen[i];
    if (l == -INFINITY) {
      s[i] = 0.f;
    } else if (SIGMOID) {
      const float q = pow2_float(-__fmul_rn(fabsf(l), LOG2E), -126.f);
      s[i] = __fdiv_rn(l >= 0.f ? 1.f : q, 1.f + q);
    } else {
      s[i] = pow2_float(below_max(l, m, LOG2E), -126.f) * inv;
    }
    share[i] = s[i];
    D += s[i];
  }
  if (rule.renorm) {
    // with the weight p = s / D in place of s, since (g - gp) / D alone overflows where D is tiny
    D = lanes_sum<L>(D);
    float gp = 0.f;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      share[i] = D > 0.f ? __fdiv_rn(s[i], D) : 0.f;
      gp += g[i] * share[i];
    }
    gp = lanes_sum<L>(gp);
#pragma unroll
    for (int i = 0; i < KL; ++i) g[i] -= gp;
  }
  float gs = 0.f;
  if (!SIGMOID && !rule.renorm) {
#pragma unroll
    for (int i = 0; i < KL; ++i) gs += g[i] * s[i];
    gs = lanes_sum<L>(gs);
  }
  T* out = dlogits + row * E;
  if (live && first < E) {
    const float q = SIGMOID ? 0.f : 0.f - gs * inv;
    if (wide_out) {
#pragma unroll
      for (int j = 0; j < V / N; ++j) {
        union {
          uint4 u;
          T t[N];
        } o;
#pragma unroll
        for (int i = 0; i < N; ++i) o.t[i] = from_f32<T>(SIGMOID ? 0.f : v[j * N + i] * q);
        reinterpret_cast<uint4*>(out + first)[j] = o.u;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (first + j < E) out[first + j] = from_f32<T>(SIGMOID ? 0.f : v[j] * q);
    }
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < KL; ++i)
    if (place[i] >= 0)
      out[place[i]] = from_f32<T>(SIGMOID ? g[i] * share[i] * (1.f - s[i]) : share[i] * (g[i] - gs));
}

// calls f(L, V) for the fewest lanes that hold E experts, eight a lane up to 256
template <class F>
erc_status with_lanes(int E, F&& f) {
  using I8 = std::integral_constant<int, 8>;
  using I16 = std::integral_constant<int, 16>;
  using I32 = std::integral_constant<int, 32>;
  if (E <= 64) return f(I8(), I8());
  if (E <= 128) return f(I16(), I8());
  if (E <= 256) return f(I32(), I8());
  if (E <= 512) return f(I32(), I16());
  return f(I32(), I32());
}
template <class T>
bool aligned16(const T* p, int64_t stride, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || stride * sizeof(T) % 16 == 0);
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
    const T* x = static_cast<const T*>(logits);
    cudaStream_t s = as_stream(stream);
    const bool grouped = rule->groups > 1 && rule->top_groups < rule->groups;
    return with_lanes(rule->experts, [&](auto l, auto v) {
      constexpr int L = decltype(l)::value, V = decltype(v)::value;
      const int size = rule->experts / rule->groups, span = size / V;
      if (grouped && (size % V || (span & (span - 1)))) {
        // groups that no power of two of lanes holds: the row in shared memory
        const size_t sh = QW * (2 * rule->experts + rule->groups) * sizeof(float);
        k_route<T><<<(unsigned)((rows + QW - 1) / QW), QW * 32, sh, s>>>(rows, x, stride, bias, *rule,
                                                                         experts, weights);
      } else if constexpr (L == 32) {
        const bool wide = aligned16(x, stride, rows) && rule->experts % V == 0;
        const int64_t most = 4LL * sm_count(), need = (rows + FW - 1) / FW;
        auto kernel = rule->score == ERC_SCORE_SIGMOID ? k_route_warp<T, V, true>
                                                       : k_route_warp<T, V, false>;
        kernel<<<(unsigned)(need < most ? need : most), FW * 32, 0, s>>>(rows, x, stride, bias, *rule,
                                                                         wide, experts, weights);
      } else {
        const bool wide = aligned16(x, stride, rows) && rule->experts % V == 0;
        const int64_t per = FW * (32 / L);
        auto kernel = rule->score == ERC_SCORE_SIGMOID ? k_route_lanes<T, L, V, true>
                                                       : k_route_lanes<T, L, V, false>;
        kernel<<<(unsigned)((rows + per - 1) / per), FW * 32, 0, s>>>(rows, x, stride, bias, *rule,
                                                                      wide, experts, weights);
      }
      count_launches(1);
      ERC_CUDA(cudaGetLastError());
      return ERC_OK;
    });
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
    const T* x = static_cast<const T*>(logits);
    T* dx = static_cast<T*>(dlogits);
    return with_lanes(rule->experts, [&](auto l, auto v) {
      constexpr int L = decltype(l)::value, V = decltype(v)::value;
      const bool even = rule->experts % V == 0;
      const bool wide = even && aligned16(x, stride, rows);
      const bool wide_out = even && aligned16(dx, rule->experts, rows);
      const int64_t per = FW * (32 / L);
      auto kernel = rule->score == ERC_SCORE_SIGMOID ? k_route_lanes_backward<T, L, V, true>
                                                     : k_route_lanes_backward<T, L, V, false>;
      kernel<<<(unsigned)((rows + per - 1) / per), FW * 32, 0, as_stream(stream)>>>(
          rows, x, stride, experts, dweights, *rule, wide, wide_out, dx);
      count_launches(1);
      ERC_CUDA(cudaGetLastError());
      return ERC_OK;
    });
  });
}
