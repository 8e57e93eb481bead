// score_rows.cu -- log probability of a given entry of each row of scores, the row's entropy and its
// best entries, and the scores' gradient.
//
// With c = log2(e) / temperature, m the largest score and t = (l - m) c, Z = sum 2^t and u = sum 2^t t
// give ln Z and the entropy ln Z - ln2 u / Z.  A part of a row (at most 48 KB) arrives in shared
// memory by one asynchronous copy; a first pass finds its maximum, a second its sums, so an entry costs one
// exponential and no part scales its sums.  Parts join by d = (m_part - m) c: u <- 2^d (u + d Z), Z <- 2^d Z.
// t is kept above -1000, where 2^t is 0, so that no product of 0 and infinity appears.
//
// The best entries: the k-th largest of the threads' maxima, found by halving, bounds the k-th best entry from
// below, so only the few entries from it on are ranked.  Where many are equal, the k-th best key and the last index
// that belongs are found the same way among all entries.
//
// Up to 8 parts are a cluster, whose first block joins them through distributed shared memory; more go
// through a workspace and a second kernel.  Short rows take 8 to 32 lanes each, rows by the thousand without best
// entries a warp each, all in registers.
//
// What bounds them: an entry costs 3 to 4 instructions, 0.3 of the time that bfloat16 rows take to arrive, and one of the
// 16 exponentials an SM makes a clock, 0.7 of it; a block's phases (copy, maximum, sums, search) wait for each other, and
// a few long rows are latency (launch, copy, two passes, the search, two cluster barriers).  Device time (us) and floor at 6767 GB/s:
//   64 x 169343 bf16, 20 best  18.4 / 3.2, none 12.4 / 3.2; 1 x 20000 f32, 5 best 8.2, none 4.8; 16384 x 257 f32, none
//   8 to 10 / 2.5, 32 best 30; 4096 x 20000 bf16, none 42 / 24.2; 3000 x 300000 bf16, none 375 / 266; 8 x 2449029 f32, none
//   24 / 11.6, 32 best 48 / 11.6.  A warp a row (4096 x 20000) issues in 0.49 of the cycles with 0.37 of the warps that fit.
// The gradient reads and writes each entry once: 4096 x 20000 bf16 53 to 56 us, 0.87 to 0.92 of the copy rate; rows whose
// result is aligned otherwise than the scores (4096 x 19999) 71 us.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int ST = 256;          // threads of a block
constexpr int SW = ST / 32;      // its warps
constexpr int SV = 4;            // vectors a lane holds at a time in the gradient
constexpr int SEGS = 96;         // segments of a block's part of a row, at most
constexpr int MAX_PARTS = 512;   // parts of a row, at most
constexpr int CLUSTER = 8;       // parts that a cluster joins, at most
constexpr int KMAX = ERC_SCORE_MAX_K;
constexpr float LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.402823466e38f;
constexpr unsigned MASKED_KEY = 0x007fffffu;  // order_key(-inf): keys up to it are no entries

__device__ __forceinline__ float exp2_fast(float t) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
  return r;
}
__device__ __forceinline__ float scaled(float l, float m, float c) {
  return l == m ? 0.f : fmaxf((l - m) * c, -1000.f);
}

// Entries met so far: `top` of them equal the largest, m (LOWEST where nothing was met); X is the sum of 2^t and u that of
// 2^t t over the others.  Z = top + X: kept apart, so that ln Z, which is X where one entry has nearly all of
// the probability, keeps its relative accuracy.
struct Sum {
  float m, X, u, top;
};
// X is NaN where a copy did not land, and stays so however parts join: everything about the row is NaN then.
__device__ __forceinline__ bool lost_row(const Sum& a) { return a.X != a.X; }
__device__ __forceinline__ float log_sum(const Sum& a) {
  return a.top > 0.f || lost_row(a) ? log1pf(a.X + (a.top - 1.f)) : -INFINITY;
}
__device__ __forceinline__ void raise(Sum& a, float m, float c) {
  if (a.m == m) return;
  const float d = scaled(a.m, m, c), f = exp2_fast(d), Z = a.X + a.top;
  a.u = f * fmaf(d, Z, a.u);
  a.X = f * Z;
  a.top = 0.f;
  a.m = m;
}
__device__ __forceinline__ Sum join(Sum a, Sum b, float c) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m, c);
  raise(b, m, c);
  return {m, a.X + b.X, a.u + b.u, a.top + b.top};
}
__device__ __forceinline__ Sum from_lane(const Sum& a, int lane) {
  return {__shfl_sync(0xffffffffu, a.m, lane), __shfl_sync(0xffffffffu, a.X, lane), __shfl_sync(0xffffffffu, a.u, lane),
          __shfl_sync(0xffffffffu, a.top, lane)};
}
// the parts of `width` neighbouring lanes joined
__device__ __forceinline__ Sum lane_join(Sum a, float c, int width) {
  for (int o = width / 2; o; o >>= 1)
    a = join(a, from_lane(a, (threadIdx.x & 31) ^ o), c);  // the same on both sides: sums and maxima commute
  return a;
}
// the largest score of a warp, and a sum over it
__device__ __forceinline__ float warp_max(float v) {
  return order_value(__reduce_max_sync(0xffffffffu, order_key(v)));
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The terms of entries whose maximum m is known (a warp that streams a row: the anchor, at most 2^1 below it).
// t = l c - fl(m c) is one fma, for two entries at once; the rounding of m c moves every t by the same d = m c - fl(m c),
// which `settle` takes out again.  Masked entries and NaN are raised to `low`, about 1000 / c below m, where 2^t is 0: one
// maximum of the stored type.  Rows where that does not hold (a maximum or a scale that is infinite, far from 0 or out of the type's
// range) take the terms one by one.
struct Scale {
  float m, c, minus_mc, low;
  bool plain;  // packed terms do
  __device__ __forceinline__ Scale(float m_, float c_) : m(m_), c(c_) {
    minus_mc = -__fmul_rn(m, c);
    low = m - __fdividef(1000.f, c);
    plain = fabsf(minus_mc) < 1e4f && c > 0.1f && c < 1e4f && low > -6e4f;
  }
};
// a vector's entries, raised to low, as pairs
__device__ __forceinline__ void raised_pairs(uint4 v, float low, uint64_t* p, float) {
  p[0] = pair(fmaxf(__uint_as_float(v.x), low), fmaxf(__uint_as_float(v.y), low));
  p[1] = pair(fmaxf(__uint_as_float(v.z), low), fmaxf(__uint_as_float(v.w), low));
}
__device__ __forceinline__ void raised_pairs(uint4 v, float low, uint64_t* p, __nv_bfloat16) {
  const __nv_bfloat162 l = __float2bfloat162_rn(low);
  const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), l);
    const unsigned b = *reinterpret_cast<const unsigned*>(&h);
    p[i] = pair(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
  }
}
__device__ __forceinline__ void raised_pairs(uint4 v, float low, uint64_t* p, __half) {
  const __half2 l = __float2half2_rn(low);
  const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(__hmax2(*reinterpret_cast<const __half2*>(&w[i]), l));
    p[i] = pair(f.x, f.y);
  }
}
struct Terms {
  uint64_t X = 0, u = 0;  // two sums each
  float top = 0.f;
};
// one entry, which may equal `top`, the largest; masked: -inf
__device__ __forceinline__ void add_entry(Terms& a, float l, const Scale& s, float top) {
  const bool largest = l == top;
  const float t = s.plain ? fmaf(fmaxf(l, s.low), s.c, s.minus_mc) : scaled(l, s.m, s.c);
  const float e = largest ? 0.f : exp2_fast(t);
  a.top += largest ? 1.f : 0.f;
  a.X = add2(a.X, pair(e, 0.f));
  a.u = fma2(pair(e, 0.f), pair(t, 0.f), a.u);
}
// holds_top: an entry that equals `top` may be among them (the largest; the anchor, where none is given)
template <class T>
__device__ __forceinline__ void add_vector(Terms& a, uint4 v, const Scale& s, bool holds_top, float top) {
  constexpr int P = ScoreVec<T>::N / 2;
  if (s.plain) {
    uint64_t l[P];
    raised_pairs(v, s.low, l, T());
    if (holds_top) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const uint64_t t = fma2(l[i], pair(s.c, s.c), pair(s.minus_mc, s.minus_mc));
        float t0, t1, l0, l1;
        unpair(t, t0, t1);
        unpair(l[i], l0, l1);
        const bool top0 = l0 == top, top1 = l1 == top;
        const uint64_t e = pair(top0 ? 0.f : exp2_fast(t0), top1 ? 0.f : exp2_fast(t1));
        a.top += (top0 ? 1.f : 0.f) + (top1 ? 1.f : 0.f);
        a.X = add2(a.X, e);
        a.u = fma2(e, t, a.u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const uint64_t t = fma2(l[i], pair(s.c, s.c), pair(s.minus_mc, s.minus_mc));
        float t0, t1;
        unpair(t, t0, t1);
        const uint64_t e = pair(exp2_fast(t0), exp2_fast(t1));
        a.X = add2(a.X, e);
        a.u = fma2(e, t, a.u);
      }
    }
  } else {
    float l[2 * P];
    unpack_scores(v, l, T());
#pragma unroll
    for (int i = 0; i < 2 * P; ++i) add_entry(a, l[i], s, top);
  }
}
template <class T>
__device__ __forceinline__ void add_vector(Terms& a, uint4 v, const Scale& s, bool holds_top) {
  add_vector<T>(a, v, s, holds_top, s.m);
}
// the sums of a lane, or of several, with d taken out: 2^-d (X, u - d X)
__device__ __forceinline__ Sum settle(Sum a, const Scale& s) {
  if (!s.plain) return a;
  const float d = fmaf(s.m, s.c, s.minus_mc), f = exp2_fast(-d);
  return {a.m, f * a.X, f * fmaf(-d, a.X, a.u), a.top};
}
__device__ __forceinline__ Sum sum_of(const Terms& a, float m) {
  float X0, X1, u0, u1;
  unpair(a.X, X0, X1);
  unpair(a.u, u0, u1);
  return {m, X0 + X1, u0 + u1, a.top};
}

struct ScoreOut {
  const int32_t* ids;
  float* logp;
  float* entropy;
  float* norm;
  int32_t* top_ids;
  float* top_logp;
  float temperature, c;
  int k;
  unsigned polls;  // looks at a copy before its block gives up (0: a second or so)
};

__device__ __forceinline__ float log_p(float l, float m, float lnZ, float temperature) {
  return l == -INFINITY ? -INFINITY : (l == m ? 0.f : __fdiv_rn(l - m, temperature)) - lnZ;
}

// a row's id, and its score (read before the sums are known)
struct Given {
  int32_t id;
  float l;
};
template <class T>
__device__ __forceinline__ Given given_of(const ScoreOut& o, int64_t row, const T* x, int64_t n) {
  Given g = {o.logp ? o.ids[row] : -1, 0.f};
  if (g.id >= 0 && g.id < n)
    g.l = clean_score(to_f32(x[g.id]));
  else
    g.id = -1;
  return g;
}
__device__ __forceinline__ void finish_row(const ScoreOut& o, int64_t row, Given g, Sum a) {
  const bool lost = lost_row(a), some = lost || a.top > 0.f;
  const float lnZ = log_sum(a), entropy = some ? lnZ - LN2 * (a.u / (a.X + a.top)) : 0.f;
  if (o.entropy) o.entropy[row] = entropy < 0.f ? 0.f : entropy;
  if (o.norm) {
    o.norm[2 * row] = lost ? NAN : some ? a.m : -INFINITY;
    o.norm[2 * row + 1] = lnZ;
  }
  if (o.logp) o.logp[row] = lost ? NAN : g.id < 0 ? 0.f : some ? log_p(g.l, a.m, lnZ, o.temperature) : -INFINITY;
}

// an entry of a row's part in the workspace
struct Best {
  unsigned key, id;
};
__device__ __forceinline__ bool ahead(unsigned ka, unsigned ia, unsigned kb, unsigned ib) {
  return ka > kb || (ka == kb && ia < ib);
}

constexpr int CAP = 256;  // entries that are ranked at once
struct TopScratch {
  Best list[CAP];
  unsigned unit[ST];  // the threads' largest keys
  unsigned least;
  int found, sum;
};

// A key that at least k of a warp's units reach (UNITS a lane; 0: none), close to the largest such one: steps down from the
// largest unit double until k are reached, six halvings follow.  MASKED_KEY + 1 where there are fewer than k.
template <int UNITS>
__device__ __forceinline__ unsigned reached_by(const unsigned* unit, int k) {
  constexpr unsigned ALL = 0xffffffffu;
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < UNITS; ++i) top = max(top, unit[i]);
  top = __reduce_max_sync(ALL, top);
  if (k == 1 || top <= MASKED_KEY) return max(top, MASKED_KEY + 1);
  auto enough = [&](unsigned t) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) c += unit[i] >= t;
    return __reduce_add_sync(ALL, c) >= k;
  };
  unsigned lo, hi = top + 1;
  for (unsigned step = 1u << 18;; step <<= 1) {
    lo = top - MASKED_KEY - 1 > step && step != 0 ? top - step : MASKED_KEY + 1;
    if (lo == MASKED_KEY + 1 || enough(lo)) break;
    hi = lo;
  }
  if (lo == MASKED_KEY + 1 && !enough(lo)) return lo;
#pragma unroll 1
  for (int i = 0; i < 6; ++i) {
    const unsigned mid = lo + (hi - lo) / 2;
    if (enough(mid)) lo = mid; else hi = mid;
  }
  return lo;
}

// the sum of a count over the block's threads
__device__ __forceinline__ int block_count(TopScratch& s, int mine) {
  mine = __reduce_add_sync(0xffffffffu, mine);
  if ((threadIdx.x & 31) == 0) atomicAdd(&s.sum, mine);
  __syncthreads();
  const int v = s.sum;
  __syncthreads();
  if (threadIdx.x == 0) s.sum = 0;
  __syncthreads();
  return v;
}

// The k best of a block's entries: each(least, f) calls f(key, id) for the thread's entries of at least that key, or for
// more; `mine` is the largest key of the thread's entries (0: none).  put(rank, key, id) takes the results, (0, 0) where
// there are fewer than k.
template <class Each, class Put>
__device__ __forceinline__ void block_top(TopScratch& s, unsigned mine, int k, Each&& each, Put&& put) {
  const int tid = threadIdx.x;
  s.unit[tid] = mine;
  if (tid == 0) s.found = s.sum = 0;
  __syncthreads();
  if (tid < 32) {
    unsigned unit[SW];
#pragma unroll
    for (int w = 0; w < SW; ++w) unit[w] = s.unit[w * 32 + tid];
    const unsigned v = reached_by<SW>(unit, k);
    if (tid == 0) s.least = v;
  }
  __syncthreads();
  const unsigned least = s.least;
  each(least, [&](unsigned key, unsigned id) {
    if (key < least) return;
    const int at = atomicAdd(&s.found, 1);
    if (at < CAP) s.list[at] = {key, id};
  });
  __syncthreads();
  int found = s.found;
  if (found > CAP) {
    unsigned edge = 0, last = 0;  // the k-th best key, and the last index that belongs among those equal to it
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned t = edge | (1u << bit);
      int c = 0;
      each(t, [&](unsigned key, unsigned) { c += key >= t; });
      if (block_count(s, c) >= k) edge = t;
    }
    int above = 0;
    each(edge, [&](unsigned key, unsigned) { above += key > edge; });
    const int need = k - block_count(s, above);
    for (int bit = 22; bit >= 0; --bit) {
      const unsigned t = last | (1u << bit);
      int c = 0;
      each(edge, [&](unsigned key, unsigned id) { c += key == edge && id < t; });
      if (block_count(s, c) < need) last = t;
    }
    if (tid == 0) s.found = 0;
    __syncthreads();
    each(edge, [&](unsigned key, unsigned id) {
      if (key > edge || (key == edge && id <= last)) s.list[atomicAdd(&s.found, 1)] = {key, id};
    });
    __syncthreads();
    found = s.found;
  }
  if (tid < found) {
    const Best b = s.list[tid];
    int before = 0;
    for (int j = 0; j < found; ++j) before += ahead(s.list[j].key, s.list[j].id, b.key, b.id);
    if (before < k) put(before, b.key, b.id);
  }
  if (tid >= found && tid < k) put(tid, 0u, 0u);
  __syncthreads();
}

__device__ __forceinline__ void put_best(const ScoreOut& o, int64_t row, Sum a, float lnZ, int rank, unsigned key,
                                         unsigned id) {
  const bool lost = lnZ != lnZ;
  o.top_ids[row * o.k + rank] = key && !lost ? (int32_t)id : -1;
  o.top_logp[row * o.k + rank] = lost ? NAN : key ? log_p(order_value(key), a.m, lnZ, o.temperature) : -INFINITY;
}

// the sums of a block whose threads share a maximum, in the order of its warps
__device__ __forceinline__ Sum block_sum(Sum a, Sum* part) {
  a.X = warp_sum(a.X);
  a.u = warp_sum(a.u);
  a.top = warp_sum(a.top);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
  __syncthreads();
  Sum all = part[0];
#pragma unroll
  for (int w = 1; w < SW; ++w) all.X += part[w].X, all.u += part[w].u, all.top += part[w].top;
  return all;
}

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t of_block(uint32_t local, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ unsigned peer_word(uint32_t at) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}

// Waits for a copy into shared memory; false when it did not land in `polls` looks at its barrier, or, with 0, in a second
// or so of waiting.
__device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity, unsigned polls) {
  uint32_t done = 0;
  if (polls == 0) {
    for (unsigned i = 0; i < (1u << 22) && !done; ++i)  // each may sleep for a while
      asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                   : "=r"(done)
                   : "r"(bar), "r"(parity)
                   : "memory");
  } else {
    for (unsigned i = 0; i < polls && !done; ++i)
      asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                   : "=r"(done)
                   : "r"(bar), "r"(parity)
                   : "memory");
  }
  return done;
}

constexpr int part_smem(int per, bool top) { return per * 16 + (top ? (int)sizeof(TopScratch) : 0); }

// A block takes one of the `parts` of a row, `per` vectors each (a multiple of 32).  CLUSTERED: the parts of a row are a
// cluster.  Blocks start with a task and take every gridDim.x-th one.  Once a copy did not land in time the block starts
// no more and gives NaN for this and its later tasks: that copy may still write the shared memory, and its barrier's
// phase is open.  The block waits for it, with a limit, before it ends.
template <class T, bool TOP, bool CLUSTERED>
__global__ void __launch_bounds__(ST) k_score_part(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                   int parts, int per, ScoreOut o, Sum* __restrict__ sums,
                                                   Best* __restrict__ best) {
  constexpr int N = ScoreVec<T>::N;
  __shared__ Sum part[SW];
  __shared__ Sum joined;
  __shared__ float top_of[SW];
  __shared__ Best kept[KMAX];
  __shared__ __align__(8) uint64_t bar_word;
  extern __shared__ __align__(16) char smem[];
  uint4* held = reinterpret_cast<uint4*>(smem);
  TopScratch& top = *reinterpret_cast<TopScratch*>(smem + per * 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t bar = shared_at(&bar_word);
  if (tid == 0) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  uint32_t parity = 0;
  bool ok = true;  // the same for all threads
  const int64_t tasks = rows * parts;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t row = task / parts;
    const int which = (int)(task - row * parts);
    const T* x = logits + row * stride;
    const RowView<T> view(x, n);
    const int first = which * per, count = max(min(per, view.vectors - first), 0);
    // whole vectors arrive by the copy, those that the row shares with its neighbours element by element
    const int lo = min(first == 0 && view.skew ? 1 : 0, count), hi = max(min(first + count, view.whole()) - first, lo);
    if (ok && tid == 0) {
      if (hi > lo) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the part before was written and read by threads
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((hi - lo) * 16) : "memory");
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_at(held + lo)),
            "l"(reinterpret_cast<const uint4*>(view.base) + first + lo), "r"((hi - lo) * 16), "r"(bar)
            : "memory");
      }
      if (lo == 1) held[0] = view.fetch(first);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (ok && tid == 32) {
      for (int v = hi; v < count; ++v) held[v] = view.fetch(first + v);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    Given g = {-1, 0.f};
    if (tid == 0 && (CLUSTERED ? which == 0 : parts == 1)) g = given_of(o, row, x, n);
    if (ok && hi > lo) {
      ok = landed(bar, parity, o.polls);
      parity ^= 1;
    }
    ok = __syncthreads_and(ok);

    const int live = ok ? count : 0;
    float m = -INFINITY;
    for (int at = tid; at < live; at += ST) m = fmaxf(m, max_score(held[at], T()));
    const unsigned mine = order_key(__fadd_rn(m, 0.f));
    const float own = m;
    m = warp_max(fmaxf(m, LOWEST));
    if (lane == 0) top_of[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SW; ++w) m = fmaxf(m, top_of[w]);
    const Scale scale(m, o.c);
    Terms terms;
    for (int at = tid; at < live; at += ST) {
      const uint4 v = held[at];
      add_vector<T>(terms, v, scale, own == m && max_score(v, T()) == m);
    }
    Sum a = settle(block_sum(sum_of(terms, m), part), scale);
    if (!ok) a = {m, NAN, NAN, NAN};
    if (TOP) {
      const bool alone = !CLUSTERED && parts == 1;
      const float lnZ = alone ? log_sum(a) : 0.f;
      block_top(
          top, mine, o.k,
          [&](unsigned least, auto&& f) {
            for (int at = tid; at < live; at += ST) {
              const uint4 v = held[at];
              if (order_key(__fadd_rn(max_score(v, T()), 0.f)) < least) continue;
              float s[N];
              unpack_scores(v, s, T());
#pragma unroll
              for (int i = 0; i < N; ++i) f(order_key(__fadd_rn(s[i], 0.f)), (unsigned)((first + at) * N + i - view.skew));
            }
          },
          [&](int rank, unsigned key, unsigned id) {
            if (CLUSTERED)
              kept[rank] = {key, id};
            else if (alone)
              put_best(o, row, a, lnZ, rank, key, id);
            else
              best[task * o.k + rank] = {key, id};
          });
    }
    if constexpr (CLUSTERED) {
      if (tid == 0) joined = a;
      cluster_sync_all();
      if (which == 0) {
        Sum all = {LOWEST, 0.f, 0.f, 0.f};
        if (lane < parts) {
          const uint32_t at = of_block(shared_at(&joined), lane);
          all = {__uint_as_float(peer_word(at)), __uint_as_float(peer_word(at + 4)), __uint_as_float(peer_word(at + 8)),
                 __uint_as_float(peer_word(at + 12))};
        }
        all = from_lane(lane_join(all, o.c, CLUSTER), 0);
        if (tid == 0) finish_row(o, row, g, all);
        if (TOP) {
          const float lnZ = log_sum(all);
          Best one = {0u, 0u};  // parts * k entries, at most one a thread
          if (tid < parts * o.k) {
            const uint32_t at = of_block(shared_at(&kept[tid % o.k]), tid / o.k);
            one = {peer_word(at), peer_word(at + 4)};
          }
          block_top(
              top, one.key, o.k, [&](unsigned, auto&& f) { f(one.key, one.id); },
              [&](int rank, unsigned key, unsigned id) { put_best(o, row, all, lnZ, rank, key, id); });
        }
      }
      cluster_sync_all();
    } else {
      if (tid == 0) {
        if (parts == 1)
          finish_row(o, row, g, a);
        else
          sums[task] = a;
      }
      __syncthreads();
    }
  }
  if (!ok) landed(bar, parity ^ 1, 0);
}

// a block joins the parts of a row
template <class T, bool TOP>
__global__ void __launch_bounds__(ST) k_score_join(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                   int parts, ScoreOut o, const Sum* __restrict__ sums,
                                                   const Best* __restrict__ best) {
  __shared__ Sum part[SW];
  extern __shared__ __align__(16) char smem[];
  TopScratch& top = *reinterpret_cast<TopScratch*>(smem);
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    Given g = {-1, 0.f};
    if (threadIdx.x == 0) g = given_of(o, row, logits + row * stride, n);
    Sum a = {LOWEST, 0.f, 0.f, 0.f};
    for (int p = threadIdx.x; p < parts; p += ST) a = join(a, sums[row * parts + p], o.c);
    a = lane_join(a, o.c, 32);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int w = 1; w < SW; ++w) a = join(a, part[w], o.c);
    if (threadIdx.x == 0) finish_row(o, row, g, a);
    if (TOP) {
      const float lnZ = log_sum(a);
      // the parts' best first, then their second best, ..: a thread's largest is some part's best, or nearly so
      const Best* from = best + row * parts * o.k;
      auto nth = [&](int i) { return from[i % parts * o.k + i / parts]; };
      unsigned mine = 0;
#pragma unroll 8
      for (int i = threadIdx.x; i < parts * o.k; i += ST) mine = max(mine, nth(i).key);
      block_top(
          top, mine, o.k,
          [&](unsigned, auto&& f) {
            for (int i0 = threadIdx.x; i0 < parts * o.k; i0 += 8 * ST) {  // eight reads in flight
              Best b[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) b[j] = i0 + j * ST < parts * o.k ? nth(i0 + j * ST) : Best{0u, 0u};
#pragma unroll
              for (int j = 0; j < 8; ++j) f(b[j].key, b[j].id);
            }
          },
          [&](int rank, unsigned key, unsigned id) { put_best(o, row, a, lnZ, rank, key, id); });
    }
    __syncthreads();
  }
}

// A warp takes a row of any length, 8 vectors a lane in flight, without a barrier.  No best entries.
//
// Terms are relative to an anchor that the largest entry so far, the peak, exceeds by at most 2^1: a higher peak turns
// the entries that equalled the one before into terms, and only where it leaves the anchor behind are the sums scaled, by less
// than 1/2, so that the roundings of many such steps add up to less than two.  A lane sums the terms of 4 rounds, 128 of a
// 16-bit type, one by one; these sums go to a second one that keeps its rounding errors, so that no row is too long (4194304
// entries would be 65536 terms to a sum: ln Z off by 5e-4).
template <class T>
__global__ void __launch_bounds__(ST, 4) k_score_stream(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                        ScoreOut o) {
  constexpr int V = 8, ROUNDS = 4;
  __shared__ float4 settled[ST];  // the second sums, X and u and the roundings of both: registers are short
  float4& held = settled[threadIdx.x];
  const int lane = threadIdx.x & 31;
  for (int64_t row = ((int64_t)blockIdx.x * ST + threadIdx.x) >> 5; row < rows; row += (int64_t)gridDim.x * SW) {
    const T* x = logits + row * stride;
    const RowView<T> view(x, n);
    Given g = {-1, 0.f};
    if (lane == 0) g = given_of(o, row, x, n);
    held = {0.f, 0.f, 0.f, 0.f};
    Scale scale(LOWEST, o.c);               // of the anchor
    float peak = LOWEST;
    Terms terms;  // its `top` counts the entries that equal the peak
    auto put_by = [&] {
      const Sum s = settle(sum_of(terms, scale.m), scale);
      const float2 X = df_two_sum(held.x, s.X), u = df_two_sum(held.y, s.u);
      held = {X.x, u.x, held.z + X.y, held.w + u.y};
      terms.X = terms.u = 0;
    };
    for (int v0 = 0; v0 < view.vectors; v0 += 32 * V) {
      uint4 v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int at = v0 + j * 32 + lane;
        v[j] = at < view.vectors ? view.fetch(at)
                                 : make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
      }
      float m = peak, best[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        best[j] = max_score(v[j], T());
        m = fmaxf(m, best[j]);
      }
      m = warp_max(m);
      if (m > peak) {
        const float t = scale.plain ? fmaf(peak, scale.c, scale.minus_mc) : scaled(peak, scale.m, scale.c);
        const float e = terms.top * exp2_fast(t);
        terms.X = add2(terms.X, pair(e, 0.f));
        terms.u = fma2(pair(e, 0.f), pair(t, 0.f), terms.u);
        terms.top = 0.f;
        peak = m;
        if (!(scaled(m, scale.m, scale.c) <= 1.f)) {
          put_by();
          const float d = scaled(scale.m, m, scale.c), f = exp2_fast(d);
          held = {f * held.x, f * fmaf(d, held.x, held.y), f * held.z, f * fmaf(d, held.z, held.w)};
          scale = Scale(m, o.c);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) add_vector<T>(terms, v[j], scale, best[j] == peak, peak);
      if (v0 / (32 * V) % ROUNDS == ROUNDS - 1) put_by();
    }
    put_by();
    Sum a = {scale.m, warp_sum(held.x + held.z), warp_sum(held.y + held.w), 0.f};
    raise(a, peak, o.c);
    a.top = warp_sum(terms.top);
    if (lane == 0) finish_row(o, row, g, a);
  }
}

// a row as whole aligned vectors, and the few entries before and behind them
template <class T>
struct ShortRow {
  const uint4* whole;
  int vectors, head, tail, tail_at;  // entries before the vectors, behind them, and where those start
  __device__ __forceinline__ ShortRow(const T* row, int n) {
    constexpr int N = ScoreVec<T>::N;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = skew ? min(N - skew, n) : 0;
    vectors = (n - head) / N;
    tail_at = head + vectors * N;
    tail = n - tail_at;
    whole = reinterpret_cast<const uint4*>(row + head);
  }
};

constexpr int SHORT_CAP = 128;

// LANES neighbouring lanes take a row of at most LANES VPL whole vectors (LANES = 32 with TOP)
template <class T, int LANES, int VPL, bool TOP>
__global__ void __launch_bounds__(ST, TOP ? 3 : 4) k_score_short(int64_t rows, int64_t n, const T* __restrict__ logits,
                                                                 int64_t stride, ScoreOut o) {
  constexpr int N = ScoreVec<T>::N;
  constexpr int EACH = ST / LANES;  // rows of a block
  constexpr unsigned ALL = 0xffffffffu;
  __shared__ Best list[TOP ? SW : 1][SHORT_CAP];
  __shared__ int found[SW];
  const int at0 = threadIdx.x % LANES, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int64_t row0 = (int64_t)blockIdx.x * EACH; row0 < rows; row0 += (int64_t)gridDim.x * EACH) {
    const int64_t row = min(row0 + threadIdx.x / LANES, rows - 1);  // a group without a row of its own repeats the last
    const bool mine = row0 + threadIdx.x / LANES < rows;
    const T* x = logits + row * stride;
    const ShortRow<T> view(x, (int)n);
    uint4 v[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int at = j * LANES + at0;
      v[j] = at < view.vectors ? __ldg(view.whole + at)
                               : make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
    }
    const float head = at0 < view.head ? clean_score(to_f32(x[at0])) : -INFINITY;
    const float tail = at0 < view.tail ? clean_score(to_f32(x[view.tail_at + at0])) : -INFINITY;
    Given g = {-1, 0.f};
    if (at0 == 0) g = given_of(o, row, x, n);
    float m = fmaxf(fmaxf(head, tail), LOWEST), peak[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      peak[j] = max_score(v[j], T());
      m = fmaxf(m, peak[j]);
    }
#pragma unroll
    for (int w = LANES / 2; w; w >>= 1) m = fmaxf(m, __shfl_xor_sync(ALL, m, w));
    const Scale scale(m, o.c);
    Terms terms;
#pragma unroll
    for (int j = 0; j < VPL; ++j) add_vector<T>(terms, v[j], scale, peak[j] == m);
    add_entry(terms, head, scale, m);
    add_entry(terms, tail, scale, m);
    Sum a = sum_of(terms, m);
#pragma unroll
    for (int w = LANES / 2; w; w >>= 1) {
      a.X += __shfl_xor_sync(ALL, a.X, w);
      a.u += __shfl_xor_sync(ALL, a.u, w);
      a.top += __shfl_xor_sync(ALL, a.top, w);
    }
    a = settle(a, scale);
    if (at0 == 0 && mine) finish_row(o, row, g, a);
    if constexpr (TOP) {
      // a vector is as good as its best entry; short rows have too few vectors and take every entry
      constexpr bool ENTRIES = VPL <= 2;
      constexpr int UNITS = (ENTRIES ? VPL * N : VPL) + 2;
      const float lnZ = log_sum(a);
      const unsigned hk = order_key(head), tk = order_key(tail);
      unsigned unit[UNITS];
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        if (ENTRIES) {
          float s[N];
          unpack_scores(v[j], s, T());
#pragma unroll
          for (int i = 0; i < N; ++i) unit[j * N + i] = order_key(__fadd_rn(s[i], 0.f));
        } else {
          unit[j] = order_key(__fadd_rn(max_score(v[j], T()), 0.f));
        }
      }
      unit[UNITS - 2] = hk;
      unit[UNITS - 1] = tk;
      const unsigned least = reached_by<UNITS>(unit, o.k);
      __syncwarp();
      if (lane == 0) found[warp] = 0;
      __syncwarp();
      auto offer = [&](unsigned key, unsigned id) {
        if (key < least) return;
        const int at = atomicAdd(&found[warp], 1);
        if (at < SHORT_CAP) list[warp][at] = {key, id};
      };
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        if (!ENTRIES && unit[j] < least) continue;
        float s[N];
        unpack_scores(v[j], s, T());
#pragma unroll
        for (int i = 0; i < N; ++i) offer(order_key(__fadd_rn(s[i], 0.f)), (unsigned)(view.head + (j * 32 + lane) * N + i));
      }
      offer(hk, (unsigned)lane);
      offer(tk, (unsigned)(view.tail_at + lane));
      __syncwarp();
      const int many = found[warp];
      if (many <= SHORT_CAP) {
        for (int i = lane; i < many; i += 32) {
          const Best b = list[warp][i];
          int before = 0;
          for (int j = 0; j < many; ++j) before += ahead(list[warp][j].key, list[warp][j].id, b.key, b.id);
          if (before < o.k && mine) put_best(o, row, a, lnZ, before, b.key, b.id);
        }
        if (lane >= many && lane < o.k && mine) put_best(o, row, a, lnZ, lane, 0u, 0u);
      } else {  // many equal ones: the best that are left, one after another
        unsigned pk = ALL, pi = 0;
        for (int r = 0; r < o.k; ++r) {
          unsigned bk = 0, bi = ALL;
          auto better = [&](unsigned key, unsigned id) {
            if (key > MASKED_KEY && ahead(pk, pi, key, id) && ahead(key, id, bk, bi)) bk = key, bi = id;
          };
#pragma unroll
          for (int j = 0; j < VPL; ++j) {
            float s[N];
            unpack_scores(v[j], s, T());
#pragma unroll
            for (int i = 0; i < N; ++i) better(order_key(__fadd_rn(s[i], 0.f)), (unsigned)(view.head + (j * 32 + lane) * N + i));
          }
          better(hk, (unsigned)lane);
          better(tk, (unsigned)(view.tail_at + lane));
          pk = __reduce_max_sync(ALL, bk);
          pi = __reduce_min_sync(ALL, bk == pk ? bi : ALL);
          if (lane == 0 && mine) put_best(o, row, a, lnZ, r, pk, pi);
        }
      }
    }
  }
}

// ---- gradient: one pass over the entries
struct ScoreGrad {
  const int32_t* ids;
  const float* norm;
  const float* entropy;
  const float* dlogp;
  const float* dentropy;
  float temperature, c;
};
// With t = l c - fl(m c + ln Z log2(e)), which is log2 p but for the rounding r of the constant (the same for all
// entries), an entry's gradient is 2^t (A t + B), and g / temperature more at the given entry.
struct RowGrad {
  Scale scale;
  float shift, A, B, lnZ, g, gh, H, inv;
  int id;
  // one entry, any row
  __device__ __forceinline__ float one(float l, int i) const {
    if (l == -INFINITY) return 0.f;
    const float t = scaled(l, scale.m, scale.c), lp = fmaf(t, LN2, -lnZ);
    const float p = exp2_fast(fmaf(lnZ, -LOG2E, t));
    // at the given entry g (1 - p) = -g (e^lp - 1), which does not cancel where p is near 1
    return i == id ? inv * fmaf(-g, expm1f(lp), -p * gh * (lp + H)) : inv * (-p * fmaf(gh, lp + H, g));
  }
};
template <class T>
__device__ __forceinline__ uint4 grad_vector(uint4 v, const RowGrad& r) {
  constexpr int P = ScoreVec<T>::N / 2;
  uint64_t l[P];
  raised_pairs(v, r.scale.low, l, T());
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint64_t t = fma2(l[i], pair(r.scale.c, r.scale.c), pair(r.shift, r.shift));
    float t0, t1, q0, q1;
    unpair(t, t0, t1);
    unpair(fma2(t, pair(r.A, r.A), pair(r.B, r.B)), q0, q1);
    q0 *= exp2_fast(t0);
    q1 *= exp2_fast(t1);
    if constexpr (sizeof(T) == 4) {
      w[2 * i] = __float_as_uint(q0);
      w[2 * i + 1] = __float_as_uint(q1);
    } else {
      w[i] = pack_pair(q0, q1, T());
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// bytes `by` .. by + 15 (a multiple of the type's size) of two vectors
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int by) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (by & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (by & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const int bits = (by & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// WARPS warps (a block, or one) take `each` vectors of a row's result, SV steps of 31 WARPS or 32 WARPS at a time.  Where the result's rows are aligned otherwise than
// the scores', a result vector is two neighbouring lanes' shifted together, and 32 lanes give 31.
// SHIFT: some rows may be aligned otherwise (71 registers and not 48, so it is left out where none can be: 63 -> 55 us for
// 4096 x 20000 bf16).
template <class T, int WARPS, bool SHIFT>
__global__ void __launch_bounds__(ST, SHIFT ? 4 : 5) k_score_backward(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                       int parts, int each, ScoreGrad o, T* __restrict__ dlogits) {
  constexpr int N = ScoreVec<T>::N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part_warp = warp % WARPS;
  const int64_t tasks = rows * parts;
  for (int64_t task = (int64_t)blockIdx.x * (SW / WARPS) + warp / WARPS; task < tasks; task += (int64_t)gridDim.x * (SW / WARPS)) {
    const int64_t row = task / parts;
    const int which = (int)(task - row * parts);
    const T* x = logits + row * stride;
    T* out = dlogits + row * n;
    const RowView<T> view(x, n);
    const int skew = (int)((reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T));  // of the result
    const int vectors = (skew + (int)n + N - 1) / N;
    // result vector u starts with entry u N - skew: entry `by` of score vector u - back
    const int delta = SHIFT ? view.skew - skew : 0, back = delta < 0 ? 1 : 0, by = delta < 0 ? delta + N : delta;
    const int wide = by ? 31 : 32, step = wide * WARPS, off = part_warp * wide;
    const int first = which * each, last = min(first + each, vectors);
    uint4 v[SV];
    auto load = [&](int u0) {
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        const int at = u0 + j * step + off + lane - back;
        if (at >= 0 && at < view.vectors && u0 + j * step + off < last)
          v[j] = view.fetch(at);
        else
          v[j] = make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
      }
    };
    load(first);
    RowGrad r = {Scale(o.norm[2 * row], o.c)};
    r.lnZ = o.norm[2 * row + 1];
    r.id = o.ids ? o.ids[row] : -1;
    const float here = r.id >= 0 && r.id < n ? clean_score(to_f32(x[r.id])) : -INFINITY;
    r.g = o.dlogp && here != -INFINITY ? o.dlogp[row] : 0.f;
    r.gh = o.dentropy ? o.dentropy[row] : 0.f;
    r.H = o.dentropy ? o.entropy[row] : 0.f;
    r.inv = __frcp_rn(o.temperature);
    {
      // shift = -(m c + Z2) rounded, Z2 = ln Z log2(e); t - rest is log2 p, rest = m c + Z2 + shift
      const float mc = -r.scale.minus_mc, Z2 = r.lnZ * LOG2E, sum = mc + Z2;
      r.shift = -sum;
      const float part = sum - mc, lost = (mc - (sum - part)) + (Z2 - part);
      const float rest = fmaf(r.scale.m, r.scale.c, -mc) + lost + fmaf(r.lnZ, LOG2E, -Z2);
      const float f = exp2_fast(-rest) * r.inv;
      r.A = -f * r.gh * LN2;
      r.B = -f * fmaf(r.gh, fmaf(-rest, LN2, r.H), r.g);
      // a masked entry's t is finite and its 2^t is 0, so that its gradient is 0 unless A t + B is not a number
      r.scale.plain = r.scale.plain && fabsf(r.A) < 1e30f && fabsf(r.B) < 1e30f;
    }
    for (int u0 = first; u0 < last; u0 += SV * step) {
      if (u0 > first) load(u0);
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        if (u0 + j * step + off >= last) break;
        union Piece {
          uint4 raw;
          T t[N];
          __device__ Piece() {}
        } q;
        const int at = u0 + j * step + off + lane - back, e0 = at * N - view.skew;
        if (r.scale.plain) {
          q.raw = grad_vector<T>(v[j], r);
          if (r.g != 0.f && r.id >= e0 && r.id < e0 + N) {
            const T mine = from_f32<T>(r.one(here, r.id));
#pragma unroll
            for (int i = 0; i < N; ++i)
              if (e0 + i == r.id) q.t[i] = mine;
          }
        } else {
          float l[N];
          unpack_scores(v[j], l, T());
#pragma unroll
          for (int i = 0; i < N; ++i) q.t[i] = from_f32<T>(r.one(l[i], e0 + i));
        }
        if (SHIFT && by) {
          const uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, q.raw.x, 1), __shfl_down_sync(0xffffffffu, q.raw.y, 1),
                                        __shfl_down_sync(0xffffffffu, q.raw.z, 1), __shfl_down_sync(0xffffffffu, q.raw.w, 1));
          q.raw = shifted(q.raw, next, by * (int)sizeof(T));
        }
        const int u = u0 + j * step + off + lane, e = u * N - skew;
        if (lane >= wide || u >= last) continue;
        if (e >= 0 && e + N <= n) {
          *reinterpret_cast<uint4*>(out + e) = q.raw;
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (e + i >= 0 && e + i < n) out[e + i] = q.t[i];
        }
      }
    }
  }
}

// Parts of a row: a part fits a block's shared memory, and few rows are split over the whole machine.  A cluster joins
// its parts without a second kernel, so up to 8 parts are preferred where 8 keep two blocks an SM busy.
struct Split {
  int parts, per;  // per: vectors of a part, a multiple of 32
};
Split split_rows(int64_t rows, int64_t n, int32_t type) {
  const int N = 16 / type_bytes(type);
  const int64_t vectors = n / N + 2;  // a row that starts inside a vector ends in one more
  const int64_t segments = (vectors + 31) / 32, least = (segments + SEGS - 1) / SEGS;
  const int64_t wanted = rows < (int64_t)sm_count() * 4 ? (int64_t)sm_count() * 4 / rows : 1;
  const int64_t most = (segments + 2 * SW - 1) / (2 * SW);  // two vectors a thread at least
  int64_t parts = wanted < most ? wanted : most;
  if (parts < least) parts = least;
  if (parts > CLUSTER && least <= CLUSTER && (rows * CLUSTER >= 2 * sm_count() || parts <= 3 * CLUSTER)) parts = CLUSTER;
  if (parts > MAX_PARTS) parts = MAX_PARTS;
  const int64_t each = (segments + parts - 1) / parts;
  return {(int)((segments + each - 1) / each), (int)each * 32};
}
// Rows enough to keep the machine busy with a warp each.  A warp a row against a block a row (us, k 0): 10000 x 5001 float16
// 35 / 45, 4096 x 20001 float32 71 / 85, 3000 x 3000 bfloat16 10.3 / 14.1, 4096 x 20000 bfloat16 43 / 41.5 (no difference
// worth a rule); fewer rows leave SMs without loads in flight:
// 2500 x 20000 bfloat16 30 / 28, 1900 x 20000 26 / 23.
bool many_rows(int64_t rows) { return rows >= (int64_t)sm_count() * 18; }
bool short_rows(int64_t n, int32_t type) { return n / (16 / type_bytes(type)) <= 32 * 8; }

erc_status check_scores(int64_t rows, int64_t n, int32_t type, int64_t stride) {
  ERC_REQUIRE(rows >= 0 && rows <= 0x7fffffffLL, "rows must be in [0, 2^31)");
  ERC_REQUIRE(n >= 0 && n <= ERC_SAMPLE_ROWS_MAX_N, "n must be in [0, %d]", ERC_SAMPLE_ROWS_MAX_N);
  ERC_REQUIRE(type >= ERC_F32 && type <= ERC_F16, "bad type %d", type);
  ERC_REQUIRE(stride >= 0, "stride must be at least 0");
  return ERC_OK;
}

struct ScorePlan {
  Sum* sums;
  Best* best;
};
void plan_scores(Arena& a, ScorePlan& p, int64_t rows, int parts, int k) {
  p.sums = a.take<Sum>((size_t)rows * parts);
  p.best = a.take<Best>((size_t)rows * parts * k);
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" size_t erc_score_rows_workspace_size(int64_t rows, int64_t n, int32_t type, int32_t k) {
  if (rows < 1 || rows > 0x7fffffffLL || n < 1 || n > ERC_SAMPLE_ROWS_MAX_N || type < ERC_F32 || type > ERC_F16 ||
      k < 0 || k > ERC_SCORE_MAX_K || short_rows(n, type))
    return 0;
  const Split sp = split_rows(rows, n, type);
  if (sp.parts <= CLUSTER || (k == 0 && many_rows(rows))) return 0;
  Arena a(nullptr);
  ScorePlan p;
  plan_scores(a, p, rows, sp.parts, k);
  return a.used + 256;
}

extern "C" erc_status erc_score_rows(int64_t rows, int64_t n, const void* logits, int32_t type, int64_t stride,
                                     const int32_t* ids, float temperature, int32_t k, float* logp, float* entropy,
                                     float* norm, int32_t* top_ids, float* top_logp, void* ws, size_t ws_bytes,
                                     erc_stream stream) {
  clear_error();
  ERC_TRY(check_scores(rows, n, type, stride));
  ERC_REQUIRE(temperature >= 1.17549435e-38f && temperature <= 3.402823466e38f,
              "temperature must be finite and at least 2^-126");
  ERC_REQUIRE(k >= 0 && k <= ERC_SCORE_MAX_K, "k must be in [0, %d]", ERC_SCORE_MAX_K);
  if (rows == 0) return ERC_OK;
  ERC_REQUIRE((n == 0 || logits) && (!ids == !logp) && (k == 0 || (top_ids && top_logp)), "null pointer");
  ERC_REQUIRE(reinterpret_cast<uintptr_t>(logits) % type_bytes(type) == 0, "misaligned logits");
  const ScoreOut o = {ids, logp, entropy, norm, top_ids, top_logp, temperature, LOG2E / temperature, k,
                      wait_limit(0)};
  const cudaStream_t s = as_stream(stream);
  const bool brief = short_rows(n, type);
  const Split sp = brief ? Split{1, 0} : split_rows(rows, n, type);
  const bool stream_rows = !brief && k == 0 && many_rows(rows);
  ScorePlan p = {};
  if (sp.parts > CLUSTER && !stream_rows) {
    if (!ws || ws_bytes < erc_score_rows_workspace_size(rows, n, type, k))
      return set_error(ERC_ERR_CAPACITY, "workspace too small");
    Arena ar(reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~uintptr_t(255)));
    plan_scores(ar, p, rows, sp.parts, k);
  }
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const T* x = static_cast<const T*>(logits);
    if (brief) {
      const int64_t vectors = n / ScoreVec<T>::N, most = (int64_t)sm_count() * 64;
      auto launch = [&](auto kernel, int lanes) {
        const int64_t blocks = (rows + ST / lanes - 1) / (ST / lanes);
        kernel<<<(unsigned)(blocks < most ? blocks : most), ST, 0, s>>>(rows, n, x, stride, o);
      };
      if (k && vectors <= 32)
        launch(k_score_short<T, 32, 1, true>, 32);
      else if (k && vectors <= 64)
        launch(k_score_short<T, 32, 2, true>, 32);
      else if (k && vectors <= 128)
        launch(k_score_short<T, 32, 4, true>, 32);
      else if (k)
        launch(k_score_short<T, 32, 8, true>, 32);
      else if (vectors <= 16)
        launch(k_score_short<T, 8, 2, false>, 8);
      else if (vectors <= 32)
        launch(k_score_short<T, 8, 4, false>, 8);
      else if (vectors <= 64)
        launch(k_score_short<T, 8, 8, false>, 8);
      else if (vectors <= 128)
        launch(k_score_short<T, 16, 8, false>, 16);
      else
        launch(k_score_short<T, 32, 8, false>, 32);
      count_launches(1);
    } else if (stream_rows) {
      const int64_t blocks = (rows + SW - 1) / SW, most = (int64_t)sm_count() * 64;
      k_score_stream<T><<<(unsigned)(blocks < most ? blocks : most), ST, 0, s>>>(rows, n, x, stride, o);
      count_launches(1);
    } else {
      const int smem = part_smem(sp.per, k > 0);
      const int64_t tasks = rows * sp.parts;
      const bool together = sp.parts > 1 && sp.parts <= CLUSTER;
      auto kernel = together ? (k ? k_score_part<T, true, true> : k_score_part<T, false, true>)
                             : (k ? k_score_part<T, true, false> : k_score_part<T, false, false>);
      if (smem > 40960)
        ERC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, part_smem(SEGS * 32, true)));
      // a grid is a whole number of clusters; blocks take further tasks a grid apart, so a cluster's stay together
      const int64_t most = (int64_t)sm_count() * 64 / sp.parts * sp.parts;
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)(tasks < most ? tasks : most));
      cfg.blockDim = dim3(ST);
      cfg.dynamicSmemBytes = smem;
      cfg.stream = s;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = together ? sp.parts : 1;
      attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = together ? 1 : 0;
      ERC_CUDA(cudaLaunchKernelEx(&cfg, kernel, rows, n, x, stride, sp.parts, sp.per, o, p.sums, p.best));
      count_launches(1);
      if (sp.parts > CLUSTER) {
        const unsigned joins = (unsigned)(rows < most ? rows : most);
        (k ? k_score_join<T, true> : k_score_join<T, false>)<<<joins, ST, k ? sizeof(TopScratch) : 0, s>>>(
            rows, n, x, stride, sp.parts, o, p.sums, p.best);
        count_launches(1);
      }
    }
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}

extern "C" erc_status erc_score_rows_backward(int64_t rows, int64_t n, const void* logits, int32_t type, int64_t stride,
                                              const int32_t* ids, float temperature, const float* norm,
                                              const float* entropy, const float* dlogp, const float* dentropy,
                                              void* dlogits, erc_stream stream) {
  clear_error();
  ERC_TRY(check_scores(rows, n, type, stride));
  ERC_REQUIRE(temperature >= 1.17549435e-38f && temperature <= 3.402823466e38f,
              "temperature must be finite and at least 2^-126");
  if (rows == 0 || n == 0) return ERC_OK;
  ERC_REQUIRE(logits && norm && dlogits && (!dlogp || ids) && (!dentropy || entropy), "null pointer");
  ERC_REQUIRE((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(dlogits)) % type_bytes(type) == 0,
              "misaligned logits or dlogits");
  const ScoreGrad o = {ids, norm, entropy, dlogp, dentropy, temperature, LOG2E / temperature};
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    // a block takes a row, or a share of one where rows are few; a warp takes a short one
    const int64_t vectors = n / ScoreVec<T>::N + 2;
    const bool wide = vectors > 31 * SV * 2;
    const int64_t unit = 31 * SV * (wide ? SW : 1), steps = (vectors + unit - 1) / unit;
    const int64_t wanted = ((int64_t)sm_count() * 8 + rows - 1) / rows;
    const int64_t parts = steps < wanted ? steps : wanted, each = (steps + parts - 1) / parts * unit;
    const int64_t tasks = rows * parts, blocks = wide ? tasks : (tasks + SW - 1) / SW, most = (int64_t)sm_count() * 256;
    const uintptr_t apart = reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits);
    const bool shift = apart % 16 != 0 || (rows > 1 && (stride - n) * (int64_t)sizeof(T) % 16 != 0);
    auto kernel = wide ? (shift ? k_score_backward<T, SW, true> : k_score_backward<T, SW, false>)
                       : (shift ? k_score_backward<T, 1, true> : k_score_backward<T, 1, false>);
    kernel<<<(unsigned)(blocks < most ? blocks : most), ST, 0, as_stream(stream)>>>(
        rows, n, static_cast<const T*>(logits), stride, (int)parts, (int)each, o, static_cast<T*>(dlogits));
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
