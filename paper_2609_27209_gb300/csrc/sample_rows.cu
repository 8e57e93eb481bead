// sample_rows.cu -- one exact draw per row of scores: temperature, min-p, top-k and top-p, then the
// inverse distribution function at a given 64-bit random word.
//
// With integer weights w_i (choice.cuh) every filter is a threshold in the order (score descending,
// index ascending): the kept set is {score > theta} and the first `ties` entries at theta.  A row's
// draw is the first kept index whose inclusive weight sum in index order exceeds floor(x W / 2^64).
#include "choice.cuh"

namespace erc {
namespace {

constexpr int RT = 512;  // threads of a row's block
constexpr int RW = RT / 32;

struct RowRule {
  float scale;               // log2(e) / T
  unsigned long long least;  // smallest eligible weight (min-p), at least 1
  unsigned top_k;            // 0xffffffff: off
  unsigned part;             // floor(top_p 2^31); 0xffffffff: off
};

__device__ __forceinline__ RowRule row_rule(const erc_sample_rule& r, int64_t row) {
  const float heat = r.temperature_rows ? r.temperature_rows[row] : r.temperature;
  const int32_t k = r.top_k_rows ? r.top_k_rows[row] : r.top_k;
  const float p = r.top_p_rows ? r.top_p_rows[row] : r.top_p;
  const float mp = r.min_p_rows ? r.min_p_rows[row] : r.min_p;
  const bool greedy = !(heat > 0.f);
  RowRule o;
  o.scale = greedy ? 1.f : __fdiv_rn(LOG2E, heat);
  o.top_k = greedy ? 1u : k > 0 ? (unsigned)k : 0xffffffffu;
  o.part = p < 1.f ? (unsigned)(fmaxf(p, 0.f) * 2147483648.f) : 0xffffffffu;
  const unsigned long long least =
      mp > 0.f ? (unsigned long long)(fminf(mp, 1.f) * 1099511627776.f) : 0ull;
  o.least = least ? least : 1ull;
  return o;
}

template <class V>
__device__ __forceinline__ V block_sum(V v, V* part) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  V s = 0;
#pragma unroll
  for (int i = 0; i < RW; ++i) s += part[i];
  return s;
}

// exclusive sum over the block's threads; *total receives the block's sum
template <class V>
__device__ __forceinline__ V block_exclusive(V v, V* part, V* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  V x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  V base = 0, all = 0;
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    if (i == warp) base = all;
    all += part[i];
  }
  *total = all;
  return base + x - v;
}

template <class T>
__global__ void __launch_bounds__(RT) k_sample_rows(int64_t n, const T* __restrict__ logits,
                                                    int64_t stride,
                                                    const uint64_t* __restrict__ words,
                                                    erc_sample_rule rule, int32_t* __restrict__ ids,
                                                    float* __restrict__ logp,
                                                    int32_t* __restrict__ kept) {
  __shared__ unsigned long long mass[256];
  __shared__ unsigned count[256];
  __shared__ unsigned long long part64[RW];
  __shared__ unsigned part32[RW];
  __shared__ unsigned s_digit, s_count;
  __shared__ unsigned long long s_mass;
  __shared__ int s_found;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * stride;
  const RowRule r = row_rule(rule, row);

  float m = -INFINITY;
  for (int64_t i = tid; i < n; i += RT) m = fmaxf(m, clean_score(to_f32(x[i])));
  {
    unsigned k = order_key(m);
    k = __reduce_max_sync(0xffffffffu, k);
    if ((tid & 31) == 0) part32[tid >> 5] = k;
    __syncthreads();
    for (int i = 0; i < RW; ++i) k = max(k, part32[i]);
    m = order_value(k);
    __syncthreads();
  }
  if (m == -INFINITY) {
    if (tid == 0) {
      ids[row] = -1;
      logp[row] = -INFINITY;
      kept[row] = 0;
    }
    return;
  }
  auto weight = [&](float l) -> unsigned long long {
    if (l == -INFINITY) return 0ull;
    const unsigned long long w = fixed_weight(below_max(l, m, r.scale));
    return w >= r.least ? w : 0ull;
  };

  // radix descent, eight bits of the key at a time: theta is the key at which the running count
  // (top-k) or the running mass (top-p) over larger entries reaches its bound
  unsigned theta = 0, ties = 0xffffffffu;
  if (r.top_k != 0xffffffffu) {
    unsigned prefix = 0, left = r.top_k;
    bool all = false;
    for (int shift = 24; shift >= 0 && !all; shift -= 8) {
      for (int b = tid; b < 256; b += RT) count[b] = 0;
      __syncthreads();
      for (int64_t i = tid; i < n; i += RT) {
        const float l = clean_score(to_f32(x[i]));
        const unsigned key = order_key(l);
        if ((shift == 24 || (key >> (shift + 8)) == prefix) && weight(l))
          atomicAdd(&count[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        unsigned c = 0;
        int b = 255;
        for (; b >= 0 && c + count[b] < left; --b) c += count[b];
        s_found = b >= 0;
        s_digit = b < 0 ? 0 : b;
        s_count = c;
      }
      __syncthreads();
      all = !s_found;
      prefix = prefix << 8 | s_digit;
      left -= s_count;
      __syncthreads();
    }
    if (!all) {
      theta = prefix;
      ties = left;
    }
  }
  if (r.part != 0xffffffffu) {
    // entries at theta all weigh the same, so top-k's own cut is a bound on their number
    unsigned long long above = 0, tied = 0, wt = 0;
    for (int64_t i = tid; i < n; i += RT) {
      const float l = clean_score(to_f32(x[i]));
      const unsigned key = order_key(l);
      const unsigned long long w = weight(l);
      if (key > theta) above += w;
      else if (key == theta && w) ++tied;
    }
    above = block_sum(above, part64);
    tied = block_sum(tied, part64);
    if (tied > ties) tied = ties;
    if (tied) wt = weight(order_value(theta));
    const unsigned long long total = above + tied * wt;
    const unsigned long long want =
        (total >> 31) * r.part + (((total & 0x7fffffffull) * r.part) >> 31);
    const unsigned long long target = want ? want : 1ull;
    if (above < target) {
      const unsigned long long need = (target - above + wt - 1) / wt;
      if (need < ties) ties = (unsigned)need;
    } else {
      unsigned prefix = 0;
      unsigned long long left = target;
      for (int shift = 24; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += RT) mass[b] = 0;
        __syncthreads();
        for (int64_t i = tid; i < n; i += RT) {
          const float l = clean_score(to_f32(x[i]));
          const unsigned key = order_key(l);
          if (key > theta && (shift == 24 || (key >> (shift + 8)) == prefix)) {
            const unsigned long long w = weight(l);
            if (w) atomicAdd(&mass[(key >> shift) & 255], w);
          }
        }
        __syncthreads();
        if (tid == 0) {
          unsigned long long c = 0;
          int b = 255;
          for (; b > 0 && c + mass[b] < left; --b) c += mass[b];
          s_digit = b;
          s_mass = c;
        }
        __syncthreads();
        prefix = prefix << 8 | s_digit;
        left -= s_mass;
        __syncthreads();
      }
      theta = prefix;
      wt = weight(order_value(theta));
      ties = (unsigned)((left + wt - 1) / wt);
    }
  }

  // the kept entries in index order: their total, then the draw
  unsigned long long total = 0;
  unsigned number = 0;
  int found = -1;
  unsigned long long at = 0, mine = 0;
  for (int pass = 0; pass < 2; ++pass) {
    unsigned long long before = 0;
    unsigned tied = 0, some = 0;
    for (int64_t base = 0; base < n; base += RT) {
      const int64_t i = base + tid;
      const float l = i < n ? clean_score(to_f32(x[i])) : -INFINITY;
      const unsigned key = order_key(l);
      unsigned long long w = key >= theta ? weight(l) : 0ull;
      unsigned all;
      const unsigned mytie = w && key == theta;
      const unsigned rank = tied + block_exclusive(mytie, part32, &all);
      tied += all;
      if (mytie && rank >= ties) w = 0;
      unsigned long long sum;
      const unsigned long long ex = before + block_exclusive(w, part64, &sum);
      if (pass == 1 && w && ex <= at && at < ex + w) {
        found = (int)i;
        mine = w;
      }
      before += sum;
      some += w != 0;
    }
    if (pass == 0) {
      total = before;
      number = block_sum(some, part32);
      at = __umul64hi(words[row], total);
    }
  }
  if (found >= 0) {
    ids[row] = found;
    kept[row] = (int32_t)number;
    const unsigned long long rest = total - mine;
    logp[row] = mine > rest ? log1pf(-__fdiv_rn(__ull2float_rn(rest), __ull2float_rn(total)))
                            : logf(__fdiv_rn(__ull2float_rn(mine), __ull2float_rn(total)));
  }
}

}  // namespace
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
    k_sample_rows<T><<<(unsigned)rows, RT, 0, as_stream(stream)>>>(
        n, static_cast<const T*>(logits), stride, words, *rule, ids, logp, kept);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
