// sample_rows.cuh -- one exact draw per row of scores: temperature, min-p, top-k and top-p, then the
// inverse distribution function at a given 64-bit random word.
//
// With integer weights w_i (choice.cuh) every filter is a threshold in the order (score descending,
// index ascending): the kept set is {score > theta} and the first `ties` entries at theta.  A row's
// draw is the first kept index whose inclusive weight sum in index order exceeds floor(x W / 2^64).
#pragma once

#include <atomic>
#include <type_traits>

#include "choice.cuh"

namespace erc {
namespace {

constexpr int SMALL = 16384;   // longest row of a block of 128 threads
constexpr int MAX_C = 16;     // blocks of a row's cluster
constexpr int CODE_LOW = 103 << 7, CODE_HIGH = 134 << 7;  // bfloat16 codes of 2^-24 and 2^7
constexpr int CODE_ZERO = CODE_HIGH - CODE_LOW + 1;        // place of 0 in the table
constexpr int CODES = 8192;   // its length; 2 CODE_ZERO + 1 places can be met
constexpr int CODES_FROM = 8192;  // shortest row that is worth a table
constexpr int DEPTH = 6;      // stages of a warp's ring of vectors
constexpr int ring_bytes(int threads) { return threads / 32 * DEPTH * 512; }

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

// The blocks of a row: a thread-block cluster, or (SOLO) one block, for which the cluster's barrier
// and remote accesses become the block's own.
template <bool SOLO>
struct Team {
  int blocks;
  unsigned rank;
  __device__ __forceinline__ explicit Team(int C) : blocks(SOLO ? 1 : C), rank(0) {
    if (!SOLO) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  }
  __device__ __forceinline__ int size() const { return SOLO ? 1 : blocks; }
  __device__ __forceinline__ void barrier() const {
    if (SOLO)
      __syncthreads();
    else
      asm volatile(
          "barrier.cluster.arrive.release.aligned;\n\t"
          "barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  // the same shared variable in block `at`
  __device__ __forceinline__ static unsigned address(const void* local, unsigned at) {
    unsigned a = (unsigned)__cvta_generic_to_shared(local), r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(at));
    return r;
  }
  __device__ __forceinline__ unsigned load(const unsigned* p, unsigned at) const {
    if (SOLO) return *p;
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(address(p, at)) : "memory");
    return v;
  }
  __device__ __forceinline__ uint4 load(const uint4* p, unsigned at) const {
    if (SOLO) return *p;
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(address(p, at))
                 : "memory");
    return v;
  }
  __device__ __forceinline__ unsigned long long load(const unsigned long long* p,
                                                     unsigned at) const {
    if (SOLO) return *p;
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(address(p, at)) : "memory");
    return v;
  }
};

// exclusive sum over the block's threads; *total receives the block's sum
template <class V, int RW>
__device__ __forceinline__ V block_exclusive(V v, V (&part)[RW], V* total) {
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
  V s = lane < RW ? part[lane] : V(0);
#pragma unroll
  for (int o = 1; o < RW; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  *total = __shfl_sync(0xffffffffu, s, RW - 1);
  const V base = __shfl_sync(0xffffffffu, s, warp ? warp - 1 : 0);
  return (warp ? base : V(0)) + x - v;
}

// The same for several values of each thread, in the order (value, thread); v becomes the sums before.
template <class V, int SEG, int RW>
__device__ __forceinline__ V block_exclusive(V (&v)[SEG], V (&part)[SEG][RW]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  V x[SEG];
#pragma unroll
  for (int g = 0; g < SEG; ++g) {
    x[g] = v[g];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const V y = __shfl_up_sync(0xffffffffu, x[g], o);
      if (lane >= o) x[g] += y;
    }
  }
  __syncthreads();
  if (lane == 31) {
#pragma unroll
    for (int g = 0; g < SEG; ++g) part[g][warp] = x[g];
  }
  __syncthreads();
  V run = 0;
#pragma unroll
  for (int g = 0; g < SEG; ++g) {
    V s = lane < RW ? part[g][lane] : V(0);
#pragma unroll
    for (int o = 1; o < RW; o <<= 1) {
      const V y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    const V base = __shfl_sync(0xffffffffu, s, warp ? warp - 1 : 0);
    v[g] = run + (warp ? base : V(0)) + x[g] - v[g];
    run += __shfl_sync(0xffffffffu, s, RW - 1);
  }
  return run;
}

struct Part {  // what a stretch of the row holds: mass and number above theta, entries at theta
  unsigned long long mass;
  unsigned above, tied;
};

template <int THREADS>
struct Shared {
  static constexpr int RT = THREADS;     // threads of a block
  static constexpr int RW = THREADS / 32;  // its warps
  // blocks of 128 threads take rows of at most SMALL entries, several an SM
  static constexpr bool LARGE = THREADS > 128;
  static constexpr int LIST = LARGE ? 8192 : 2048;   // candidates listed in a block's memory
  static constexpr int RANK = LARGE ? 4096 : 1024;   // candidates of a row that one block ranks
  static constexpr int TINY = LARGE ? 256 : 128;     // candidates drawn from one a thread
  static constexpr int BIN_BITS = LARGE ? 10 : 9;    // of the bins of one level of the descent
  static constexpr int BINS = 1 << BIN_BITS;
  static constexpr int STEPS = LARGE ? 128 : 16;     // bins an octave of the weights' histogram
  static constexpr int WBINS = 32 * STEPS;           // its bins
  static constexpr int CBINS = LARGE ? 1024 : 256;   // bins of the threads' maxima
  unsigned long long part64[RW], mass[RW], total64, sure64;
  unsigned part32[RW], above[RW], tied[RW];
  unsigned long long sub_mass[RW];  // of the parts of the drawn region
  unsigned sub_tied[RW];
  unsigned top, low;          // the block's largest entry and smallest thread maximum, as keys
  unsigned number;            // candidates of this block
  unsigned theta, ties, some; // what block 0 decided from the list
  unsigned digit;             // a level's bin
  unsigned first_bin, last_bin;  // of the weights' histogram
  unsigned long long over;    // a level's sum before that bin
  unsigned odd;               // entries that the code table has no place for
  static constexpr int SEG = LARGE ? CODES / (4 * RT) : 1;  // fours of places of a thread
  unsigned long long seg64[SEG][RW];
  unsigned seg32[SEG][RW];
  union {
    struct {
      union {
        unsigned bins[3][BINS];
        unsigned count[CBINS];
        alignas(16) unsigned wbins[WBINS];
      };
      unsigned list[LIST];    // candidates' keys
      uint8_t from[LIST];     // and the warps whose regions hold them
    };
    alignas(16) unsigned codes[LARGE ? CODES : 4];  // entries of each bfloat16 code, then its 2^t if it is kept
  };
};

template <class T>
struct Row {
  static constexpr int N = ScoreVec<T>::N;
  RowView<T> view;
  uint4* ring;  // DEPTH stages of 32 vectors for each warp
  int first, last, region;  // this block's vectors, and vectors of a warp's region
  float max, scale;
  bool odd;  // a maximum of +inf or an infinite scale
  unsigned long long least;
  float tmin;  // entries with t below this weigh less than `least`

  // with the maximum set: the row's scale and eligibility
  __device__ __forceinline__ void rules(const RowRule& rule) {
    scale = rule.scale;
    least = rule.least;
    odd = max == INFINITY || scale > 3.4028234e38f;
    tmin = rule.least <= 1 ? -41.5f : log2f((float)rule.least - 0.5f) - 40.01f;
  }
  __device__ __forceinline__ int begin(int warp) const { return first + warp * region; }
  __device__ __forceinline__ int end(int warp) const { return min(last, begin(warp) + region); }
  __device__ __forceinline__ void scores(uint4 u, float* l) const { unpack_scores(u, l, T()); }
  __device__ __forceinline__ float scaled(float l) const {
    return odd ? below_max(l, max, scale) : __fmul_rn(__fsub_rn(l, max), scale);
  }
  __device__ __forceinline__ bool eligible(float l) const {
    const float t = scaled(l);
    if (!(t >= tmin)) return false;
    return (least <= 1 && t > -40.9f) || weight(l);  // t near the edge is weighed
  }
  // the weight of a score, 0 if it is not eligible
  __device__ __forceinline__ unsigned long long weight(float l) const {
    if (l == -INFINITY) return 0ull;
    const unsigned long long w = fixed_weight(below_max(l, max, scale));
    return w >= least ? w : 0ull;
  }
};

// f(vector, its number) for vectors [from, to) of the row, 32 at a time (lanes past the end get masked
// vectors).
// Each lane's vectors arrive in the warp's ring of shared memory, DEPTH - 1 ahead, and are read by
// that lane alone.
template <class T, class F>
__device__ __forceinline__ void each_vector(const Row<T>& r, int from, int to, F&& f) {
  const int lane = threadIdx.x & 31;
  auto masked = [] {
    const unsigned w = masked_word<T>();
    return make_uint4(w, w, w, w);
  };
  if (from == 0 && r.view.skew) {  // the first vector is shared with the row before
    f(lane < to ? r.view.fetch(lane) : masked(), lane);
    from = 32;
  }
  const int whole = min(to, r.view.whole());  // vectors up to here are the row's own
  const uint4* src = reinterpret_cast<const uint4*>(r.view.base) + (from + lane);
  const unsigned ring = (unsigned)__cvta_generic_to_shared(
      r.ring + (threadIdx.x >> 5) * (DEPTH * 32) + lane);
  const int ahead = whole - 32 * (DEPTH - 1);
  auto issue = [&](bool own, unsigned at, const uint4* p) {
    if (own) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(p) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d)
    issue(from + lane + 32 * d < whole, ring + d * 512, src + 32 * d);
  unsigned stage = ring, last = ring + (DEPTH - 1) * 512;
  src += 32 * (DEPTH - 1);
  int v = from + lane;
  for (int left = to - from; left > 0; left -= 32, v += 32, src += 32) {
    issue(v < ahead, last, src);
    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
    uint4 u;
    if (v < whole)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                   : "r"(stage)
                   : "memory");
    else
      u = v < to ? r.view.fetch(v) : masked();
    f(u, v);
    last = stage;
    stage = stage == ring + (DEPTH - 1) * 512 ? ring : stage + 512;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// mass, numbers and ties of vectors [from, to), over the lanes
template <class T>
__device__ Part measure(const Row<T>& r, int from, int to, float theta) {
  constexpr int N = Row<T>::N;
  Part p = {0, 0, 0};
  unsigned hi = 0, lo = 0, parts = 0;
  if (r.least == 1 && theta == -INFINITY && !r.odd) {
    const uint64_t m2 = pair(-r.max, -r.max), s2 = pair(r.scale, r.scale);
    each_vector(r, from, to, [&](uint4 u, int) {
      uint64_t l[N / 2];
      unpack_pairs<T>(u, l);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        float t[2], v[2];
        unsigned h[2], w[2];
        unpair(mul2(add2(l[i], m2), s2), t[0], t[1]);
        weight_parts(t[0], t[1], h, w, v);
        hi += h[0] + h[1];
        lo += w[0] + w[1];
        p.above += (v[0] >= 0x1p-41f) + (v[1] >= 0x1p-41f);
      }
      parts += N;
    });
  } else {
    each_vector(r, from, to, [&](uint4 u, int) {
      const float best = max_score(u, T());
      if (!(best >= theta) || !(r.scaled(best) >= r.tmin)) return;
      float l[N];
      r.scores(u, l);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        unsigned h[2], w[2];
        float v[2], t[2];
        if (!(fmaxf(l[i], l[i + 1]) >= theta)) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) t[j] = l[i + j] > theta ? r.scaled(l[i + j]) : -60.f;
        if (!(fmaxf(t[0], t[1]) >= r.tmin) && theta == -INFINITY) continue;
        weight_parts(t[0], t[1], h, w, v);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (r.least <= 1) {
            hi += h[j];
            lo += w[j];
            ++parts;
            p.above += v[j] >= 0x1p-41f;
          } else {
            const unsigned long long x = join_parts(h[j], w[j]);
            p.mass += x >= r.least ? x : 0ull;
            p.above += x >= r.least;
          }
          p.tied += l[i + j] == theta && theta > -INFINITY;  // theta itself is eligible
        }
      }
    });
  }
  if (parts) p.mass += join_sums(hi, lo, parts);
  p.above = __reduce_add_sync(0xffffffffu, p.above);
  p.tied = __reduce_add_sync(0xffffffffu, p.tied);
#pragma unroll
  for (int o = 16; o; o >>= 1) p.mass += __shfl_xor_sync(0xffffffffu, p.mass, o);
  return p;
}

// The row's kept mass by warps of the cluster: every thread i < C * RW gets the place of warp i's
// region in it.  theta = -inf: no threshold.
struct Measured {
  unsigned long long before, kept, total, above_mass;
  unsigned ties_before, number, tied;
};
template <class T, bool SOLO, class S>
__device__ Measured by_regions(S& s, const Row<T>& r, const Team<SOLO>& team, float theta,
                               unsigned ties) {
  constexpr int RW = S::RW;
  const int C = team.size();
  const int tid = threadIdx.x;
  team.barrier();
  Part q = {0, 0, 0};
  if (tid < C * RW) {
    q.mass = team.load(&s.mass[tid % RW], tid / RW);
    q.above = team.load(&s.above[tid % RW], tid / RW);
    q.tied = team.load(&s.tied[tid % RW], tid / RW);
  }
  Measured m;
  unsigned tied, above;
  m.ties_before = block_exclusive(q.tied, s.part32, &tied);
  block_exclusive(q.above, s.part32, &above);
  block_exclusive(q.mass, s.part64, &m.above_mass);
  m.kept = q.mass;
  if (q.tied && m.ties_before < ties)
    m.kept += min(q.tied, ties - m.ties_before) * r.weight(theta);
  m.before = block_exclusive(m.kept, s.part64, &m.total);
  m.tied = tied;
  m.number = above + min(tied, ties);
  return m;
}
template <class T, bool SOLO, class S>
__device__ Measured measure_row(S& s, const Row<T>& r, const Team<SOLO>& team, float theta,
                                unsigned ties) {
  const int warp = threadIdx.x >> 5;
  const Part p = measure(r, r.begin(warp), r.end(warp), theta);
  if ((threadIdx.x & 31) == 0) {
    s.mass[warp] = p.mass;
    s.above[warp] = p.above;
    s.tied[warp] = p.tied;
  }
  return by_regions(s, r, team, theta, ties);
}

// f(score, warp of its region) for the entries of the block that are no lower than `floor`: those of
// its regions, or (LISTED) of its candidate list
template <bool LISTED, class T, class F, class S>
__device__ __forceinline__ void each_score(const S& s, const Row<T>& r, float floor, F&& f) {
  constexpr int RT = S::RT;
  constexpr int N = Row<T>::N;
  const int tid = threadIdx.x, warp = tid >> 5;
  if (LISTED) {
    for (unsigned i = tid; i < s.number; i += RT) {
      const float l = order_value(s.list[i]);
      if (l >= floor) f(l, s.from[i]);
    }
    return;
  }
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
    if (max_score(u, T()) >= floor) {
      float l[N];
      r.scores(u, l);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (l[i] >= floor) f(l[i], warp);
    }
  });
}

// Descent to the key at which the running count (MASS: weight) over entries with keys in
// [klo, khi] and t of at most `limit`, largest first, reaches `left` (> 0).  Returns false where it does not; else khi is
// that key and `left` what is still wanted from the entries at it.  A level splits the keys into
// at most BINS bins; a bin's weights are summed as three limbs of 14 bits, at most 2^18 of them in
// a block, and the blocks of the cluster each add up a part of the bins.
template <bool MASS, bool LISTED, class T, bool SOLO, class S>
__device__ bool descend(S& s, const Row<T>& r, const Team<SOLO>& team, unsigned klo,
                        unsigned& khi, unsigned long long& left, float limit = INFINITY) {
  constexpr int RT = S::RT;
  const int C = team.size();
  const unsigned rank = team.rank;
  const int tid = threadIdx.x;
  const int B = S::BINS / C;
  for (;;) {
    const unsigned span = khi - klo;
    const int shift = span < S::BINS ? 0 : 32 - S::BIN_BITS - __clz(span);
    for (int b = tid; b < (MASS ? 3 : 1) * S::BINS; b += RT) s.bins[0][b] = 0;
    __syncthreads();
    each_score<LISTED>(s, r, order_value(klo), [&](float l, int) {
      const unsigned d = khi - order_key(__fadd_rn(l, 0.f));
      const bool in = d <= span && (LISTED || limit == INFINITY || r.scaled(l) <= limit);
      const unsigned long long w = in ? r.weight(l) : 0ull;
      if (w) {
        const unsigned b = d >> shift;
        if (MASS) {
          atomicAdd(&s.bins[0][b], (unsigned)w & 0x3fff);
          atomicAdd(&s.bins[1][b], (unsigned)(w >> 14) & 0x3fff);
          atomicAdd(&s.bins[2][b], (unsigned)(w >> 28));
        } else {
          atomicAdd(&s.bins[0][b], 1u);
        }
      }
    });
    team.barrier();
    // this block's share of the bins: bins rank * B .., BINS / RT of them a thread at most
    unsigned long long v[S::BINS / RT], mine = 0;
    const int per = (B + RT - 1) / RT;
#pragma unroll
    for (int i = 0; i < S::BINS / RT; ++i) {
      v[i] = 0;
      const int b = tid * per + i;
      if (i < per && b < B)
        for (int c = 0; c < C; ++c) {
          v[i] += team.load(&s.bins[0][rank * B + b], c);
          if (MASS)
            v[i] += ((unsigned long long)team.load(&s.bins[1][rank * B + b], c) << 14) +
                    ((unsigned long long)team.load(&s.bins[2][rank * B + b], c) << 28);
        }
      mine += v[i];
    }
    unsigned long long sum;
    unsigned long long before = block_exclusive(mine, s.part64, &sum);
    if (tid == 0) s.total64 = sum;
    team.barrier();
    unsigned long long base = 0;
    int owner = -1;
    for (int c = 0; c < C; ++c) {
      const unsigned long long q = team.load(&s.total64, c);
      if (owner < 0) {
        if (base + q >= left) owner = c;
        else base += q;
      }
    }
    if (owner == (int)rank) {
      before += base;
#pragma unroll
      for (int i = 0; i < S::BINS / RT; ++i) {
        if (v[i] && before < left && left <= before + v[i]) {
          s.digit = rank * B + tid * per + i;
          s.over = before;
        }
        before += v[i];
      }
    }
    team.barrier();
    if (owner < 0) return false;
    const unsigned digit = team.load(&s.digit, owner);
    left -= team.load(&s.over, owner);
    khi -= digit << shift;
    const unsigned width = (1u << shift) - 1;
    if (khi - klo > width) klo = khi - width;
    team.barrier();
    if (klo == khi) return true;
  }
}

struct RowOut {  // where a row's result goes, and its word
  uint64_t word;
  int32_t* id;
  float* logp;
  int32_t* kept;
  __device__ __forceinline__ void set(int index, unsigned long long w, unsigned long long total,
                                      unsigned number) const {
    const unsigned long long rest = total - w;
    *id = index;
    *kept = (int32_t)number;
    *logp = w > rest ? log1pf(-__fdiv_rn(__ull2float_rn(rest), __ull2float_rn(total)))
                     : logf(__fdiv_rn(__ull2float_rn(w), __ull2float_rn(total)));
  }
  __device__ __forceinline__ void none() const {
    *id = -1;
    *logp = -INFINITY;
    *kept = 0;
  }
};

// The draw from at most TINY candidates, one a thread: ranked by counting, filtered in that order,
// and drawn by counting again in the order of their indices.
template <class T, class S>
__device__ void draw_tiny(S& s, const Row<T>& r, const RowRule& rule, unsigned all,
                          const RowOut& out) {
  const unsigned tid = threadIdx.x;
  unsigned long long* order = reinterpret_cast<unsigned long long*>(s.wbins);  // (key, ~index)
  unsigned long long* weights = order + S::TINY;                              // by rank
  unsigned* index = reinterpret_cast<unsigned*>(weights + S::TINY);
  const unsigned mine = tid < all ? s.list[S::RANK + tid] : 0u;
  const unsigned long long own =
      tid < all ? (unsigned long long)s.list[tid] << 32 | (0xffffffffu - mine) : 0ull;
  if (tid < all) order[tid] = own;
  __syncthreads();
  if (tid < all) {
    unsigned rank = 0;
    for (unsigned j = 0; j < all; ++j) rank += order[j] > own;
    weights[rank] = r.weight(order_value((unsigned)(own >> 32)));
    index[rank] = mine;
  }
  __syncthreads();
  const unsigned keep = min(all, rule.top_k);
  const unsigned long long w = tid < keep ? weights[tid] : 0ull;
  unsigned long long total;
  const unsigned long long before = block_exclusive(w, s.part64, &total);
  unsigned long long target = ~0ull;
  if (rule.part != 0xffffffffu) {
    target = (total >> 31) * rule.part + (((total & 0x7fffffffull) * rule.part) >> 31);
    if (!target) target = 1;
  }
  const bool in = w && before < target;
  const unsigned number = __syncthreads_count(in);  // the first `number` ranks
  if (in && tid == number - 1) s.over = before + w;
  __syncthreads();
  if (in) {
    const unsigned long long at = __umul64hi(out.word, s.over);
    unsigned long long earlier = 0;
    const unsigned here = index[tid];
    for (unsigned j = 0; j < number; ++j)
      if (index[j] < here) earlier += weights[j];
    if (at >= earlier && at - earlier < w) out.set((int)here, w, s.over, number);
  }
}

// Ranks at most RANK candidates in block 0: top-k, then top-p, to (theta, ties).  Candidates are the
// eligible entries whose distance from the maximum is below `reach` (all of them: reach = inf).
// At most TINY of them are drawn from right there, which ends the row.
enum Ranked { TOO_MANY, RANKED, DRAWN };
template <class T, bool SOLO, class S>
__device__ Ranked rank_list(S& s, const Row<T>& r, const RowRule& rule, const Team<SOLO>& team,
                            float inv, float reach, float& theta, unsigned& ties,
                            const RowOut& out) {
  constexpr int RT = S::RT;
  constexpr int N = Row<T>::N;
  const int C = team.size();
  const unsigned rank = team.rank;
  const int tid = threadIdx.x, warp = tid >> 5;
  unsigned* index = s.list + S::RANK;  // of the candidates
  if (tid == 0) s.number = 0;
  __syncthreads();
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int at) {
    const float best = max_score(u, T());
    if (!(__fmul_rn(__fsub_rn(r.max, best), inv) < reach)) return;
    float l[N];
    r.scores(u, l);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (__fmul_rn(__fsub_rn(r.max, l[i]), inv) < reach && r.eligible(l[i])) {
        const unsigned p = atomicAdd(&s.number, 1u);
        if (p < S::RANK) {
          s.list[p] = order_key(__fadd_rn(l[i], 0.f));
          index[p] = at * N - r.view.skew + i;
        }
      }
  });
  team.barrier();
  unsigned all = 0, mine = 0;
  for (int c = 0; c < C; ++c) {
    const unsigned q = team.load(&s.number, c);
    if (c == 0) mine = q;
    all += q;
  }
  if (all > S::RANK) {
    team.barrier();
    return TOO_MANY;
  }
  if (rank == 0) {
    unsigned at = mine;
    for (int c = 1; c < C; ++c) {
      const unsigned q = team.load(&s.number, c);
      for (unsigned i = tid; i < q; i += RT) {
        s.list[at + i] = team.load(&s.list[i], c);
        index[at + i] = team.load(&index[i], c);
      }
      at += q;
    }
    __syncthreads();
  }
  if (all <= S::TINY) {
    if (rank == 0) draw_tiny(s, r, rule, all, out);
    return DRAWN;
  }
  if (rank == 0) {
    unsigned size = 2;
    while (size < all) size *= 2;
    for (unsigned i = all + tid; i < size; i += RT) s.list[i] = 0;
    __syncthreads();
    for (unsigned k = 2; k <= size; k *= 2)  // bitonic sort, largest first
      for (unsigned j = k / 2; j; j /= 2) {
        for (unsigned i = tid; i < size / 2; i += RT) {
          const unsigned a = 2 * i - (i & (j - 1)), b = a + j;
          const unsigned x = s.list[a], y = s.list[b];
          if ((x < y) == ((a & k) == 0)) {
            s.list[a] = y;
            s.list[b] = x;
          }
        }
        __syncthreads();
      }
    // each thread takes RANK / RT consecutive candidates
    const unsigned keep = min(all, rule.top_k);
    unsigned long long w[S::RANK / RT], sum = 0, total;
#pragma unroll
    for (int i = 0; i < S::RANK / RT; ++i) {
      const unsigned at_i = tid * (S::RANK / RT) + i;
      w[i] = at_i < keep ? r.weight(order_value(s.list[at_i])) : 0ull;
      sum += w[i];
    }
    unsigned long long before = block_exclusive(sum, s.part64, &total);
    unsigned long long target = ~0ull;
    if (rule.part != 0xffffffffu) {
      target = (total >> 31) * rule.part + (((total & 0x7fffffffull) * rule.part) >> 31);
      if (!target) target = 1;
    }
    unsigned kept = 0;
#pragma unroll
    for (int i = 0; i < S::RANK / RT; ++i) {
      if (w[i] && before < target) ++kept;
      before += w[i];
    }
    unsigned number;
    block_exclusive(kept, s.part32, &number);
    if (tid == 0) {
      // (theta, ties): the last kept key, and how many of the kept ones have it
      const unsigned key = number ? s.list[number - 1] : 0u;
      unsigned lo = 0, hi = number;  // first of the kept with that key
      while (lo < hi) {
        const unsigned mid = (lo + hi) / 2;
        if (s.list[mid] > key) lo = mid + 1;
        else hi = mid;
      }
      s.theta = key;
      s.ties = number - lo;
    }
  }
  team.barrier();
  theta = order_value(team.load(&s.theta, 0));
  ties = team.load(&s.ties, 0);
  return RANKED;
}

// Sum over the cluster of a value of each thread.
template <bool SOLO, class S>
__device__ unsigned long long team_sum(S& s, unsigned long long v, unsigned long long* slot,
                                       const Team<SOLO>& team) {
  const int C = team.size();
  const int lane = threadIdx.x & 31;
  unsigned long long sum;
  block_exclusive(v, s.part64, &sum);
  if (threadIdx.x == 0) *slot = sum;
  team.barrier();
  sum = lane < C ? team.load(slot, lane) : 0ull;
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return sum;
}

// whether a block's list holds more than it can
template <bool SOLO, class S>
__device__ bool overflowed(S& s, const Team<SOLO>& team) {
  bool over = false;
  for (int k = 0; k < team.size(); ++k) over = over || team.load(&s.number, k) > S::LIST;
  return over;
}

// the keys of entries with to_t < t <= from_t, with room for the roundings of t
template <class T>
__device__ __forceinline__ void bin_keys(const Row<T>& r, float to_t, float from_t, unsigned& klo,
                                         unsigned& khi) {
  auto score_at = [&](float t, float room) {
    return __fadd_rn(r.max, __fdiv_rn(t + room, r.scale)) + room * 1e-4f * fabsf(r.max);
  };
  klo = order_key(fmaxf(score_at(to_t, -0.01f), -3.4028235e38f));
  khi = order_key(fminf(score_at(from_t, 0.01f), r.max));
}

// appends the lanes' entries to the block's list
template <class S>
__device__ __forceinline__ void append(S& s, bool in, float l, int warp) {
  const int lane = threadIdx.x & 31;
  const unsigned those = __ballot_sync(0xffffffffu, in);
  unsigned q = 0;
  if (lane == 0) q = atomicAdd(&s.number, (unsigned)__popc(those));
  q = __shfl_sync(0xffffffffu, q, 0) + __popc(those & ((1u << lane) - 1));
  if (in && q < S::LIST) {
    s.list[q] = order_key(__fadd_rn(l, 0.f));
    s.from[q] = (uint8_t)warp;
  }
}

// Top-p alone over long rows.  One pass weighs the row and counts its entries by weight, STEPS bins
// an octave: a bin's entries weigh within 0.55% of each other, so the counts bound the running mass
// from both sides and leave a few bins in which theta lies.  A second pass weighs what is above
// them, which is kept, and lists their entries; theta is found in the list (in
// the row itself where a block's list overflows).  Bins are stretches of t (floor(-t STEPS), an
// exact product), and so are all comparisons.
// `m` receives the kept row by regions (see Measured).
template <class T, bool SOLO, class S>
__device__ void nucleus(S& s, const Row<T>& r, const RowRule& rule, const Team<SOLO>& team,
                        float& theta, unsigned& ties, Measured& m) {
  constexpr int RT = S::RT;
  const int C = team.size();
  constexpr int N = Row<T>::N;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int stop = r.end(warp);
  // the maximum alone weighs 2^40: all entries below `cut` together weigh less than an eighth of
  // 1 - top_p of that, so theta is above it (or below the last bin)
  const float rest = 1.f - __fmul_rn((float)rule.part, 0x1p-31f);
  const float cut = fmaxf(log2f(__fdiv_rn(rest, (float)r.view.n)) - 3.01f, -(float)S::WBINS / S::STEPS);
  const float low = fmaxf(cut, r.tmin - 1.f);
  for (int b = tid; b < S::WBINS; b += RT) s.wbins[b] = 0;
  if (tid == 0) s.number = 0;
  __syncthreads();
  unsigned long long mass = 0;
  const uint64_t m2 = pair(-r.max, -r.max), s2 = pair(r.scale, r.scale);
  if (r.least <= 1) {
    const unsigned bins = (unsigned)__cvta_generic_to_shared(s.wbins) - (BIAS << 2);
    unsigned hi = 0, lo = 0, parts = 0;
    each_vector(r, r.begin(warp), stop, [&](uint4 u, int) {
      uint64_t l[N / 2];
      unpack_pairs<T>(u, l);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        float t[2], v[2];
        unsigned h[2], w[2];
        unpair(mul2(add2(l[i], m2), s2), t[0], t[1]);
        weight_parts(t[0], t[1], h, w, v);
        hi += h[0] + h[1];
        lo += w[0] + w[1];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const unsigned bin = __float_as_uint(__fmaf_rz(t[j], -(float)S::STEPS, 8388608.f));
          asm volatile(
              "{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], 1;\n\t}" ::"f"(t[j]),
              "f"(low), "r"(bins + (bin << 2))
              : "memory");
        }
      }
      parts += N;
    });
    if (parts) mass = join_sums(hi, lo, parts);
  } else {
    each_vector(r, r.begin(warp), stop, [&](uint4 u, int) {
      const float best = max_score(u, T());
      if (!(r.scaled(best) >= r.tmin)) return;
      float l[N];
      r.scores(u, l);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float t = r.scaled(l[i]);
        const unsigned long long w = t >= r.tmin ? r.weight(l[i]) : 0ull;
        mass += w;  // what is too light to be counted belongs to the sum all the same
        if (w && t > low) atomicAdd(&s.wbins[__float_as_uint(__fmaf_rz(t, -(float)S::STEPS, 8388608.f)) - BIAS], 1u);
      }
    });
  }
  const unsigned long long total = team_sum(s, mass, &s.total64, team);  // also closes the counting
  unsigned long long target =
      (total >> 31) * rule.part + (((total & 0x7fffffffull) * rule.part) >> 31);
  if (!target) target = 1;
  // bounds of the running mass through each bin, from the bins before it and from those after it
  float from_t, to_t;  // theta lies in to_t < t <= from_t
  {
    constexpr int P = S::WBINS / RT;
    unsigned c[P] = {};
#pragma unroll 4
    for (int k = 0; k < C; ++k)
#pragma unroll
      for (int i = 0; i < P; i += 4) {
        const uint4 q = team.load(reinterpret_cast<const uint4*>(&s.wbins[tid * P + i]), k);
        c[i] += q.x;
        c[i + 1] += q.y;
        c[i + 2] += q.z;
        c[i + 3] += q.w;
      }
    unsigned long long least[P], most[P], ls = 0, ms = 0, all_least, all_most;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float top = exp2f(40.f - (float)(tid * P + i) * (1.f / S::STEPS));
      const float bottom = top * exp2f(-1.f / S::STEPS) * (1.f - 2e-5f);
      least[i] = c[i] * (bottom > 1.f ? (unsigned long long)(bottom - 1.f) : 0ull);
      most[i] = c[i] * ((unsigned long long)(top * (1.f + 2e-5f)) + 1ull);
      ls += least[i];
      ms += most[i];
    }
    unsigned long long lb = block_exclusive(ls, s.part64, &all_least);
    unsigned long long mb = block_exclusive(ms, s.part64, &all_most);
    const unsigned long long below =  // what is not counted weighs at most this
        low > cut ? 0ull : (unsigned long long)(exp2f(40.f + low) * 1.001f * (float)r.view.n) + r.view.n;
    if (tid == 0) {
      s.first_bin = S::WBINS;
      s.last_bin = S::WBINS;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const unsigned long long l0 = lb, m0 = mb;
      lb += least[i];
      mb += most[i];
      auto upper = [&](unsigned long long most_to, unsigned long long least_to) {
        return min(most_to, total - min(total, all_least - least_to));
      };
      auto lower = [&](unsigned long long most_to, unsigned long long least_to) {
        const unsigned long long after = all_most - most_to + below;
        return max(least_to, total - min(total, after));
      };
      const bool start = tid == 0 && i == 0;
      if (upper(mb, lb) >= target && (start || upper(m0, l0) < target)) s.first_bin = tid * P + i;
      if (lower(mb, lb) >= target && (start || lower(m0, l0) < target)) s.last_bin = tid * P + i;
    }
    __syncthreads();
    from_t = -(float)s.first_bin * (1.f / S::STEPS);
    to_t = s.last_bin < S::WBINS ? -(float)(s.last_bin + 1) * (1.f / S::STEPS) : -INFINITY;
  }
  // what lies above the bins, by regions, and the list of what lies in them
  Part p = {0, 0, 0};
  {
    unsigned hi = 0, lo = 0, parts = 0;
    each_vector(r, r.begin(warp), stop, [&](uint4 u, int) {
      uint64_t l[N / 2];
      float t[N], best = -INFINITY;
      unpack_pairs<T>(u, l);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        unpair(mul2(add2(l[i], m2), s2), t[2 * i], t[2 * i + 1]);
        best = fmaxf(best, fmaxf(t[2 * i], t[2 * i + 1]));
      }
      if (!__any_sync(0xffffffffu, best > to_t)) return;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned who = __ballot_sync(0xffffffffu, t[i] <= from_t && t[i] > to_t);
        if (!who) continue;
        float x0, x1;
        unpair(l[i / 2], x0, x1);
        const float x = i & 1 ? x1 : x0;
        append(s, (who >> lane & 1) && (r.least <= 1 || r.weight(x)), x, warp);
      }
      if (!__any_sync(0xffffffffu, best > from_t)) return;
      if (r.least <= 1) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          unsigned h[2], w[2];
          float v[2];
          const bool k0 = t[i] > from_t, k1 = t[i + 1] > from_t;
          weight_parts(k0 ? t[i] : -60.f, k1 ? t[i + 1] : -60.f, h, w, v);
          hi += h[0] + h[1];
          lo += w[0] + w[1];
          p.above += k0 + k1;
        }
        parts += N;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float x0, x1;
          unpair(l[i / 2], x0, x1);
          const unsigned long long w = t[i] > from_t ? r.weight(i & 1 ? x1 : x0) : 0ull;
          p.mass += w;
          p.above += w != 0;
        }
      }
    });
    if (parts) p.mass += join_sums(hi, lo, parts);
  }
  p.above = __reduce_add_sync(0xffffffffu, p.above);
#pragma unroll
  for (int o = 16; o; o >>= 1) p.mass += __shfl_xor_sync(0xffffffffu, p.mass, o);
  if (lane == 0) {
    s.mass[warp] = p.mass;
    s.above[warp] = p.above;
    s.tied[warp] = 0;
  }
  const unsigned long long sure = team_sum(s, lane == 0 ? p.mass : 0ull, &s.sure64, team);
  const bool over = overflowed(s, team);
  team.barrier();
  // sure < target: theta is among the bins' entries
  unsigned long long left = target - sure;
  unsigned klo, khi;
  bin_keys(r, to_t, from_t, klo, khi);
  auto settle = [&](auto listed) {  // theta, and what the bins' entries add to the regions
    constexpr bool L = decltype(listed)::value;
    descend<true, L>(s, r, team, klo, khi, left, from_t);
    each_score<L>(s, r, order_value(khi), [&](float l, int region) {
      if (!L && r.scaled(l) > from_t) return;
      const unsigned long long w = r.weight(l);
      if (!w) return;
      const bool tie = order_key(__fadd_rn(l, 0.f)) == khi;
      if (!tie) atomicAdd(&s.mass[region], w);
      atomicAdd(tie ? &s.tied[region] : &s.above[region], 1u);
    });
  };
  if (over)
    settle(std::false_type());
  else
    settle(std::true_type());
  theta = order_value(khi);
  const unsigned long long wt = r.weight(theta);
  ties = (unsigned)((left + wt - 1) / wt);
  m = by_regions(s, r, team, theta, ties);
}

// Top-k with more entries than the threads' maxima can bound: a pass counts the entries by the bins
// of nucleus(), which gives the bin of the top_k-th exactly.  Where the entries down to that bin
// can be ranked, they are.  Else the bin's entries are listed and theta found among them (limited),
// which leaves top-p to the caller (TOO_MANY), as where fewer than top_k entries lie in the bins.
template <class T, bool SOLO, class S>
__device__ Ranked tally(S& s, const Row<T>& r, const RowRule& rule, const Team<SOLO>& team,
                        float& theta, unsigned& ties, bool& limited, const RowOut& out) {
  constexpr int RT = S::RT;
  constexpr int N = Row<T>::N;
  constexpr int P = S::WBINS / RT;
  const int tid = threadIdx.x, warp = tid >> 5;
  const float low = fmaxf(r.tmin - 1.f, -(float)S::WBINS / S::STEPS);
  team.barrier();  // the bins share memory with counts that other blocks read
  for (int b = tid; b < S::WBINS; b += RT) s.wbins[b] = 0;
  if (tid == 0) s.number = 0;
  __syncthreads();
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
    float l[N];
    r.scores(u, l);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = r.scaled(l[i]);
      if (t > low && (r.least <= 1 || r.eligible(l[i])))
        atomicAdd(&s.wbins[__float_as_uint(__fmaf_rz(t, -(float)S::STEPS, 8388608.f)) - BIAS], 1u);
    }
  });
  team.barrier();
  unsigned c[P] = {}, sum = 0, all;
#pragma unroll 4
  for (int k = 0; k < team.size(); ++k)
#pragma unroll
    for (int i = 0; i < P; i += 4) {
      const uint4 q = team.load(reinterpret_cast<const uint4*>(&s.wbins[tid * P + i]), k);
      c[i] += q.x;
      c[i + 1] += q.y;
      c[i + 2] += q.z;
      c[i + 3] += q.w;
    }
#pragma unroll
  for (int i = 0; i < P; ++i) sum += c[i];
  unsigned before = block_exclusive(sum, s.part32, &all);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (before < rule.top_k && rule.top_k <= before + c[i]) {
      s.first_bin = tid * P + i;
      s.some = before;
      s.digit = c[i];
    }
    before += c[i];
  }
  team.barrier();
  if (all < rule.top_k) {
    // every eligible entry, where all of them lie in the bins and can be ranked
    if (r.tmin - 1.f <= -(float)S::WBINS / S::STEPS || all > S::RANK) return TOO_MANY;
    return rank_list(s, r, rule, team, r.scale, -low, theta, ties, out);
  }
  const unsigned bin = s.first_bin;
  const float from_t = -(float)bin * (1.f / S::STEPS), to_t = -(float)(bin + 1) * (1.f / S::STEPS);
  unsigned long long left = rule.top_k - s.some;
  if (s.some + s.digit <= S::RANK)
    return rank_list(s, r, rule, team, r.scale, -to_t, theta, ties, out);
  __syncthreads();
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
    float l[N];
    r.scores(u, l);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = r.scaled(l[i]);
      if (__any_sync(0xffffffffu, t <= from_t && t > to_t))
        append(s, t <= from_t && t > to_t && r.weight(l[i]), l[i], warp);
    }
  });
  team.barrier();
  const bool over = overflowed(s, team);
  team.barrier();
  unsigned klo, khi;
  bin_keys(r, to_t, from_t, klo, khi);
  if (over)
    descend<false, false>(s, r, team, klo, khi, left, from_t);
  else
    descend<false, true>(s, r, team, klo, khi, left, from_t);
  theta = order_value(khi);
  ties = (unsigned)left;
  limited = true;
  return rule.part == 0xffffffffu ? RANKED : TOO_MANY;
}

// ------------------------------------------------------------------------------------------------
// bfloat16 rows by their codes
// ------------------------------------------------------------------------------------------------
// The 16 bits of a score say its weight, so one pass that counts the row's entries by code holds all
// that the filters need: a place of the table for every magnitude in [2^-24, 2^7) of either sign, and
// for 0, in descending order of the scores.  Each thread takes fours of places, weighs those that
// have entries, and running sums over the threads give theta and its ties exactly.  A second pass adds up
// the kept weights of each region, read from the table (as 2^t, whose parts give the integer).
// Returns 1, or 0 for a row with nothing to draw, or -1 where entries without a place of their own
// could change the result.
//
// 256 rows of 232,965, top-p: 264 us by weighing every entry twice, 142 us so (57 instructions an
// entry over both passes).

// four times the place of the bfloat16 in the upper half of `t` (a: its magnitude): 0's for magnitudes
// below the table, one past the last of their sign for those above it
__device__ __forceinline__ int code_place4(unsigned t, int& a) {
  a = (int)(t >> 16) & 0x7fff;
  const int i = min(max(a, CODE_LOW - 1), CODE_HIGH) - (CODE_LOW - 1);
  const int negative = (int)t >> 31;  // -1 or 0
  return (CODE_ZERO + ((i ^ ~negative) + 1 + negative)) << 2;
}
__device__ __forceinline__ float place_value(int place) {
  const int i = place - CODE_ZERO;
  if (i == 0) return 0.f;
  const unsigned a = (unsigned)(abs(i) + CODE_LOW - 1) << 16;
  return __uint_as_float(i > 0 ? a | 0x80000000u : a);
}

template <class T, bool SOLO, class S>
__device__ int by_codes(S& s, Row<T>& r, const RowRule& rule, const Team<SOLO>& team,
                        float& theta, unsigned& ties, Measured& m) {
  constexpr int RT = S::RT;
  constexpr int SEG = S::SEG, P = 4 * SEG;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int b = tid; b < CODES; b += RT) s.codes[b] = 0;
  if (tid == 0) {
    s.odd = 0;
    s.top = CODES;
    s.last_bin = 0;
    s.some = 0;
  }
  __syncthreads();
  auto place_of = [&](int i) { return (i / 4) * 4 * RT + tid * 4 + i % 4; };  // ascending in i
  const unsigned table = (unsigned)__cvta_generic_to_shared(s.codes);
  bool odd = false, tiny = false;
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned t = i & 1 ? w[i / 2] : w[i / 2] << 16;
      int a;
      const unsigned at = table + code_place4(t, a);
      asm volatile(
          "{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], 1;\n\t}" ::"r"(a),
          "n"(CODE_HIGH), "r"(at)
          : "memory");
      if ((unsigned)(a - CODE_LOW) >= CODE_HIGH - CODE_LOW) {  // 0, masked, or no place of its own
        tiny = tiny || (a != 0 && a < CODE_LOW);
        odd = odd || !(a < CODE_LOW || a > 0x7f80 || (t >> 16) == 0xff80);
      }
    }
  });
  if (odd) atomicOr(&s.odd, 1u);
  if (tiny) atomicOr(&s.odd, 2u);
  team.barrier();
  unsigned any = 0;
  for (int c = 0; c < team.size(); ++c) any |= team.load(&s.odd, c);
  unsigned count[P];
#pragma unroll
  for (int i = 0; i < P; ++i) count[i] = 0;
  for (int c = 0; c < team.size(); ++c)
#pragma unroll
    for (int i = 0; i < P; i += 4) {
      const uint4 q = team.load(reinterpret_cast<const uint4*>(&s.codes[place_of(i)]), c);
      count[i] += q.x;
      count[i + 1] += q.y;
      count[i + 2] += q.z;
      count[i + 3] += q.w;
    }
  unsigned first = CODES;
#pragma unroll
  for (int i = P - 1; i >= 0; --i)
    if (count[i]) first = place_of(i);
  first = __reduce_min_sync(0xffffffffu, first);
  if (lane == 0) atomicMin(&s.top, first);
  team.barrier();  // the counts have been read everywhere
  if (any & 1) return -1;
  if (s.top == CODES) return 0;
  r.max = place_value((int)s.top);
  // magnitudes below 2^-24 were counted as 0: beside a maximum of at least 2 their difference from it
  // rounds to the same float, so they weigh the same
  if (any && fabsf(r.max) < 2.f) return -1;
  r.rules(rule);

  // 2^t of each place, and its integer weight where it is eligible
  float v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = 0.f;
  auto weight = [&](float x) {
    unsigned hi[2], lo[2];
    split_weights(pair(x, x), hi, lo);
    return join_parts(hi[0], lo[0]);
  };
  unsigned entries[SEG] = {};
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (count[i]) {
      const float t = r.scaled(place_value(place_of(i)));
      v[i] = t > -41.5f ? pow2_float(t, -41.f) : 0.f;
      if (weight(v[i]) < r.least) count[i] = 0;
      entries[i / 4] += count[i];
    }
  block_exclusive(entries, s.seg32);
  auto left_by_k = [&](unsigned before, unsigned n) {
    return before < rule.top_k ? min(n, rule.top_k - before) : 0u;
  };
  unsigned long long mass[SEG] = {};
#pragma unroll
  for (int i = 0; i < P; ++i) {
    unsigned& before = entries[i / 4];
    if (count[i]) mass[i / 4] += left_by_k(before, count[i]) * weight(v[i]);
    before += count[i];
  }
  const unsigned long long total = block_exclusive(mass, s.seg64);
  unsigned long long target = ~0ull;
  if (rule.part != 0xffffffffu) {
    target = (total >> 31) * rule.part + (((total & 0x7fffffffull) * rule.part) >> 31);
    if (!target) target = 1;
  }
  unsigned number = 0, last = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (i % 4 == 0)  // back to the sums before the four places
      entries[i / 4] -= count[i] + count[i + 1] + count[i + 2] + count[i + 3];
    unsigned& before = entries[i / 4];
    unsigned long long& mass_before = mass[i / 4];
    const unsigned n = left_by_k(before, count[i]);
    float keep = 0.f;
    if (n && mass_before < target) {
      const unsigned long long w = weight(v[i]);
      unsigned kept = n;
      if (target - mass_before < n * w) kept = (unsigned)((target - mass_before + w - 1) / w);
      if (kept < count[i])
        s.some = kept;  // only the last kept place is kept in part
      else
        keep = v[i];
      number += kept;
      last = place_of(i);
      mass_before += n * w;
    }
    before += count[i];
    s.codes[place_of(i)] = __float_as_uint(keep);
  }
  last = __reduce_max_sync(0xffffffffu, last);
  if (lane == 0) atomicMax(&s.last_bin, last);
  unsigned all_kept;
  block_exclusive(number, s.part32, &all_kept);  // also orders what the block's threads wrote
  __syncthreads();
  if (any && s.some && s.last_bin == CODE_ZERO) return -1;  // but they are no ties of 0
  theta = place_value((int)s.last_bin);
  ties = s.some ? s.some : 0xffffffffu;
  // (where 0 is the last place kept, so are the smaller magnitudes below it)
  if (any && s.last_bin == CODE_ZERO) theta = -0x1.fep-25f;

  // the regions' kept mass, and their entries at a theta kept in part
  const int theta4 = s.some ? (int)s.last_bin << 2 : -1;
  Part p = {0, 0, 0};
  unsigned hi = 0, lo = 0, parts = 0;
  each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
    const float best = max_score(u, T());
    if (!(best >= theta)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int a;
      const int p0 = code_place4(w[i] << 16, a), p1 = code_place4(w[i], a);
      const float v0 = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(s.codes) + p0);
      const float v1 = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(s.codes) + p1);
      unsigned h[2], q[2];
      split_weights(pair(v0, v1), h, q);
      hi += h[0] + h[1];
      lo += q[0] + q[1];
      p.tied += (p0 == theta4) + (p1 == theta4);
    }
    parts += 8;
  });
  if (parts) p.mass = join_sums(hi, lo, parts);
  p.tied = __reduce_add_sync(0xffffffffu, p.tied);
#pragma unroll
  for (int o = 16; o; o >>= 1) p.mass += __shfl_xor_sync(0xffffffffu, p.mass, o);
  if (lane == 0) {
    s.mass[warp] = p.mass;
    s.above[warp] = 0;
    s.tied[warp] = p.tied;
  }
  m = by_regions(s, r, team, theta, ties);
  m.number = all_kept;
  return 1;
}

// The draw from the kept row: the warp's region it falls in, then a sixteenth of that region, then a
// vector.
template <class T, bool SOLO, class S>
__device__ void draw(S& s, const Row<T>& r, const Team<SOLO>& team, float theta, unsigned ties,
                     const Measured& m, const RowOut& out) {
  constexpr int RW = S::RW;
  constexpr int N = Row<T>::N;
  const int C = team.size();
  const unsigned rank = team.rank;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned long long at = __umul64hi(out.word, m.total);
  if (tid < C * RW && at >= m.before && at - m.before < m.kept) {
    s.digit = tid;
    s.over = m.before;
    s.some = m.ties_before;
  }
  __syncthreads();
  const int owner = (int)s.digit;
  if (owner / RW == (int)rank) {
    const unsigned long long wt = theta == -INFINITY ? 0ull : r.weight(theta);
    const int ow = owner % RW, ob = r.begin(ow), oe = r.end(ow);
    const int step = ((oe - ob + 31) / 32 + RW - 1) / RW * 32;  // vectors of a sixteenth
    const int from = min(oe, ob + warp * step), to = min(oe, from + step);
    unsigned long long before = s.over;
    unsigned ties_before = s.some;
    const Part p = measure(r, from, to, theta);
    if (lane == 0) {
      s.sub_mass[warp] = p.mass;
      s.sub_tied[warp] = p.tied;
    }
    __syncthreads();
    auto with_ties = [&](unsigned long long mass, unsigned tied, unsigned earlier) {
      return tied && earlier < ties ? mass + min(tied, ties - earlier) * wt : mass;
    };
    for (int w = 0; w < warp; ++w) {
      before += with_ties(s.sub_mass[w], s.sub_tied[w], ties_before);
      ties_before += s.sub_tied[w];
    }
    const unsigned long long here = with_ties(p.mass, p.tied, ties_before);
    if (at >= before && at - before < here) {  // one warp: 32 vectors at a time
      const unsigned mw = masked_word<T>();
      const uint4 masked = make_uint4(mw, mw, mw, mw);
      for (int v0 = from; v0 < to; v0 += 32) {
        float l[N];
        r.scores(v0 + lane < to ? r.view.fetch(v0 + lane) : masked, l);
        unsigned long long mass = 0;
        unsigned tied = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const unsigned long long w = l[i] >= theta ? r.weight(l[i]) : 0ull;
          if (w && l[i] == theta) ++tied;
          else mass += w;
        }
        unsigned tied_to = tied;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned y = __shfl_up_sync(0xffffffffu, tied_to, o);
          if (lane >= o) tied_to += y;
        }
        unsigned mine_before = ties_before + tied_to - tied;
        const unsigned long long k = with_ties(mass, tied, mine_before);
        unsigned long long k_to = k;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long y = __shfl_up_sync(0xffffffffu, k_to, o);
          if (lane >= o) k_to += y;
        }
        unsigned long long b = before + k_to - k;
        if (at >= b && at - b < k) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            unsigned long long w = l[i] >= theta ? r.weight(l[i]) : 0ull;
            if (w && l[i] == theta && mine_before++ >= ties) w = 0;
            if (at >= b && at - b < w) out.set((v0 + lane) * N - r.view.skew + i, w, m.total, m.number);
            b += w;
          }
        }
        before += __shfl_sync(0xffffffffu, k_to, 31);
        ties_before += __shfl_sync(0xffffffffu, tied_to, 31);
        if (at < before) break;
      }
    }
  }
}

template <class T, bool SOLO, class S>
__device__ void sample_row(S& s, Row<T>& r, const RowRule& rule, const Team<SOLO>& team,
                           const RowOut& out) {
  constexpr int RT = S::RT, RW = S::RW;
  const int C = team.size();
  const unsigned rank = team.rank;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int TM = 4;  // maxima of a thread
  const bool by_k = rule.top_k < (unsigned)r.view.n, by_p = rule.part != 0xffffffffu;
  float theta = -INFINITY;
  unsigned ties = 0xffffffffu;
  Measured m;
  if constexpr (std::is_same<T, __nv_bfloat16>::value && S::LARGE) {
    const bool k_by_maxima = by_k && rule.top_k <= (unsigned)min(RT * TM / 4 * C, 512);
    if (r.view.n >= CODES_FROM && (by_k || by_p) && !k_by_maxima) {
      const int found = by_codes(s, r, rule, team, theta, ties, m);
      if (found == 0) {
        if (rank == 0 && tid == 0) out.none();
        return;
      }
      if (found > 0) {
        draw(s, r, team, theta, ties, m, out);
        return;
      }
    }
  }

  // the row's maximum, and each thread's maxima over a quarter of its vectors
  float tm[TM];
#pragma unroll
  for (int k = 0; k < TM; ++k) tm[k] = -INFINITY;
  {
    each_vector(r, r.begin(warp), r.end(warp), [&](uint4 u, int) {
      const float best = fmaxf(tm[0], max_score(u, T()));
#pragma unroll
      for (int i = 1; i < TM; ++i) tm[i - 1] = tm[i];  // each fourth vector's maximum
      tm[TM - 1] = best;
    });
  }
  {
    unsigned hi = 0, lo = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < TM; ++k) {
      tm[k] = __fadd_rn(tm[k], 0.f);
      hi = max(hi, order_key(tm[k]));
      if (tm[k] != -INFINITY) lo = min(lo, order_key(tm[k]));
    }
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lo);
    if (lane == 0) {
      s.part32[warp] = hi;
      s.above[warp] = lo;
    }
    for (int b = tid; b < S::CBINS; b += RT) s.count[b] = 0;
    __syncthreads();
    if (warp == 0) {
      const unsigned h = __reduce_max_sync(0xffffffffu, lane < RW ? s.part32[lane] : 0u);
      const unsigned w = __reduce_min_sync(0xffffffffu, lane < RW ? s.above[lane] : 0xffffffffu);
      if (lane == 0) {
        s.top = h;
        s.low = w;
      }
    }
  }
  team.barrier();
  unsigned top = 0, low = 0xffffffffu;
  {
    const unsigned t = lane < C ? team.load(&s.top, lane) : 0u;
    const unsigned w = lane < C ? team.load(&s.low, lane) : 0xffffffffu;
    top = __reduce_max_sync(0xffffffffu, t);
    low = __reduce_min_sync(0xffffffffu, w);
  }
  r.max = order_value(top);
  if (r.max == -INFINITY) {  // the same in every block of the cluster
    if (rank == 0 && tid == 0) out.none();
    return;
  }
  r.rules(rule);

  bool done = false, limited = false, measured = false;
  if (by_k && !r.odd) {
    // At least top_k entries lie no lower than the top_k-th best of the threads' maxima: those down
    // to its bin are the candidates.
    Ranked ranked = TOO_MANY;
    const float inv = __fdiv_rn((float)(S::CBINS - 1), __fsub_rn(r.max, order_value(low)));
    if (inv < 1e30f && rule.top_k <= (unsigned)(RT * TM / 4 * C)) {
#pragma unroll
      for (int k = 0; k < TM; ++k)
        if (r.eligible(tm[k])) {
          const unsigned b = min((unsigned)(int)__fmul_rn(__fsub_rn(r.max, tm[k]), inv), S::CBINS - 1u);
          atomicAdd(&s.count[b], 1u);
        }
      team.barrier();
      unsigned c[S::CBINS / RT], sum = 0, all;
#pragma unroll
      for (int i = 0; i < S::CBINS / RT; ++i) {
        c[i] = 0;
#pragma unroll 4
        for (int q = 0; q < C; ++q) c[i] += team.load(&s.count[tid * (S::CBINS / RT) + i], q);
        sum += c[i];
      }
      unsigned before = block_exclusive(sum, s.part32, &all);
#pragma unroll
      for (int i = 0; i < S::CBINS / RT; ++i) {
        if (before < rule.top_k && rule.top_k <= before + c[i]) s.digit = tid * (S::CBINS / RT) + i;
        before += c[i];
      }
      team.barrier();
      if (all >= rule.top_k)
        ranked = rank_list(s, r, rule, team, inv, (float)s.digit + 1.f, theta, ties, out);
    }
    if (ranked == TOO_MANY) ranked = tally(s, r, rule, team, theta, ties, limited, out);
    if (ranked == DRAWN) return;
    done = ranked == RANKED;
  }
  if (!by_k && by_p && !r.odd) {
    nucleus(s, r, rule, team, theta, ties, m);
    done = measured = true;
  }
  if (!done) {
    // keys an eligible entry can have: t >= tmin, with room for its roundings
    const float edge = r.odd ? -INFINITY
                             : __fadd_rn(r.max, __fdiv_rn(r.tmin - 0.5f, r.scale)) - 1e-5f * fabsf(r.max);
    unsigned klo = order_key(fmaxf(edge, -3.4028235e38f));
    if (by_k && !limited) {
      unsigned khi = top;
      unsigned long long left = rule.top_k;
      if (descend<false, false>(s, r, team, klo, khi, left)) {
        theta = order_value(khi);
        ties = (unsigned)left;
        limited = true;
      }
    }
    if (by_p) {
      m = measure_row(s, r, team, theta, ties);
      team.barrier();
      unsigned long long target =
          (m.total >> 31) * rule.part + (((m.total & 0x7fffffffull) * rule.part) >> 31);
      if (!target) target = 1;
      if (m.above_mass < target) {
        const unsigned long long wt = r.weight(theta);
        ties = (unsigned)((target - m.above_mass + wt - 1) / wt);
      } else {
        if (limited) klo = order_key(theta) + 1;
        unsigned khi = top;
        unsigned long long left = target;
        descend<true, false>(s, r, team, klo, khi, left);
        theta = order_value(khi);
        const unsigned long long wt = r.weight(theta);
        ties = (unsigned)((left + wt - 1) / wt);
      }
    }
  }

  if (!measured) m = measure_row(s, r, team, theta, ties);
  draw(s, r, team, theta, ties, m, out);
}

// A cluster of C blocks takes a row: block c its c-th contiguous part, each of the block's warps a
// contiguous region of that, so that the index order is the order of (block, warp, vector, lane) and a
// draw is found from the regions' sums without a scan over the row.
//
// Issue-bound, not memory-bound.  256 rows of 232,965 bf16, top-p 0.95: 142 us, 0.84 TB/s of the
// row's bytes; 57 instructions an entry over both passes.  Schedulers issue in 69% of their active
// cycles, and 256 blocks leave a sixth of the machine's 304 places empty.
// 64 rows of 169,343 bf16, mixed rules: 52 us.  One row of 20,000 f32, top-k 50 and top-p: 18 us,
// latency of the call, the block scans and the cluster's barriers.
template <class T, bool SOLO, int RT>
__global__ void __launch_bounds__(RT, 1024 / RT)
    k_sample_rows(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                  const uint64_t* __restrict__ words, erc_sample_rule rule, int C,
                  int32_t* __restrict__ ids, float* __restrict__ logp, int32_t* __restrict__ kept) {
  extern __shared__ uint4 ring[];
  __shared__ Shared<RT> s;
  const Team<SOLO> team(C);
  C = team.size();
  for (int64_t row = blockIdx.x / C; row < rows; row += gridDim.x / C) {
    Row<T> r = {RowView<T>(logits + row * stride, n)};
    const int part = (r.view.vectors + C - 1) / C;
    r.ring = ring;
    r.first = min(r.view.vectors, (int)team.rank * part);
    r.last = min(r.view.vectors, r.first + part);
    r.region = (part + RT - 1) / RT * 32;
    const RowOut out = {words[row], &ids[row], &logp[row], &kept[row]};
    sample_row(s, r, row_rule(rule, row), team, out);
    team.barrier();
  }
}

// Blocks of a row.  A block holds at most 2^18 entries (sums of 14-bit limbs and of weight parts stay
// in 32 bits).  Beyond that, blocks are added to a row while the machine has room for them (two
// blocks an SM) and a block still gets 4096 entries; rows that fill the machine by themselves take
// one block each.  Passes after the first find the row in L2.
int blocks_of(int64_t rows, int64_t n) {
  int C = 1;
  while (C < MAX_C && n > ((int64_t)C << 18)) C *= 2;
  while (C < MAX_C && rows * C * 2 <= 2 * sm_count() && n >= C * 2 * 4096) C *= 2;
  return C;
}

// ------------------------------------------------------------------------------------------------
// short rows: a warp takes a row, `q` consecutive entries a lane (odd: no bank conflicts)
// ------------------------------------------------------------------------------------------------
constexpr int SW = 4;          // warps of a block
constexpr int SHORT = 1536;    // longest row (2000 entries: a block of 128 threads is faster)
constexpr int short_q(int64_t n) { return (int)((n + 31) / 32) | 1; }

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <class V>
__device__ __forceinline__ V warp_inclusive(V v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x & 31) >= o) v += y;
  }
  return v;
}

// The largest key K in [floor, top] with sum(K) >= want, where sum(K) is what entries with keys of
// at least K sum to and sum(floor) >= want: the bits below the highest one in which the two ends
// differ, one by one.
template <class F>
__device__ __forceinline__ unsigned largest_key(unsigned floor, unsigned top,
                                                unsigned long long want, F&& sum) {
  const unsigned differ = floor ^ top;
  if (!differ) return top;
  int bit = 31 - __clz(differ);
  unsigned key = top >> bit >> 1 << 1 << bit;  // the shared bits (bit may be 31)
  for (; bit >= 0; --bit) {
    const unsigned c = key | 1u << bit;
    if (c <= floor || (c <= top && sum(c) >= want)) key = c;
  }
  return key;
}

constexpr int SBINS = 256;  // bins of a warp's histogram, six an octave of the weights

// A warp's row: its entries' keys (0: not eligible), `q` consecutive ones a lane, and 2^t of each.
struct ShortRow {
  unsigned* keys;
  const float* powers;  // only where entries are weighed
  unsigned* bins;       // 2 SBINS
  unsigned* list;       // 32
  int q;
  float best, scale;  // the row's maximum and log2(e) / T

  __device__ __forceinline__ int bin(unsigned key) const {
    const float t = below_max(order_value(key), best, scale);
    return min((int)(__float_as_uint(__fmaf_rz(t, -6.f, 8388608.f)) - BIAS), SBINS - 1);
  }
  __device__ __forceinline__ unsigned long long weight(int i) const {
    unsigned hi[2], lo[2];
    split_weights(pair(powers[i], powers[i]), hi, lo);
    return join_parts(hi[0], lo[0]);
  }
  // The key at which the running count (MASS: weight) over the keys above `below`, largest first,
  // reaches `left`, which it does; `left` becomes what is still wanted from the entries at that
  // key.  A histogram gives the bin, and the bin's entries, one a lane, the key; more than 32 of them
  // are searched bit by bit.  A bin's parts of weights are sums of at most 2048: 32 bits hold them.
  template <bool MASS>
  __device__ unsigned find(unsigned below, unsigned long long& left) const {
    const int lane = threadIdx.x & 31;
    constexpr int P = SBINS / 32;
    for (int b = lane; b < (MASS ? 2 : 1) * SBINS; b += 32) bins[b] = 0;
    __syncwarp();
    for (int i = lane * q; i < (lane + 1) * q; ++i) {
      const unsigned k = keys[i];
      if (k <= below) continue;
      const int b = bin(k);
      if (MASS) {
        unsigned hi[2], lo[2];
        split_weights(pair(powers[i], powers[i]), hi, lo);
        atomicAdd(&bins[b], hi[0] - BIAS);
        atomicAdd(&bins[SBINS + b], lo[0] - BIAS);
      } else {
        atomicAdd(&bins[b], 1u);
      }
    }
    __syncwarp();
    unsigned long long v[P], sum = 0;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      v[j] = bins[lane * P + j];
      if (MASS) v[j] = (v[j] << 20) + bins[SBINS + lane * P + j];
      sum += v[j];
    }
    unsigned long long before = warp_inclusive(sum) - sum, rest = 0;
    int mine = -1;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      if (before < left && left <= before + v[j]) {
        mine = lane * P + j;
        rest = left - before;
      }
      before += v[j];
    }
    const int owner = __ffs(__ballot_sync(0xffffffffu, mine >= 0)) - 1;
    const int at = __shfl_sync(0xffffffffu, mine, owner);
    left = __shfl_sync(0xffffffffu, rest, owner);
    // the bin's entries
    unsigned number = 0, low = 0xffffffffu, high = 0;
    for (int i = lane * q; i < (lane + 1) * q; ++i) {
      const unsigned k = keys[i];
      const bool in = k > below && bin(k) == at;
      const unsigned who = __ballot_sync(0xffffffffu, in);
      const unsigned p = number + __popc(who & ((1u << lane) - 1));
      if (in) {
        if (p < 32) list[p] = i;
        low = min(low, k);
        high = max(high, k);
      }
      number += __popc(who);
    }
    __syncwarp();
    if (number <= 32) {
      const int i = (unsigned)lane < number ? (int)list[lane] : -1;
      const unsigned k = i >= 0 ? keys[i] : 0u;
      const unsigned long long w = i >= 0 ? (MASS ? weight(i) : 1ull) : 0ull;
      unsigned long long over = 0, same = 0;
      for (unsigned j = 0; j < number; ++j) {
        const unsigned ok = __shfl_sync(0xffffffffu, k, j);
        const unsigned long long ow = __shfl_sync(0xffffffffu, w, j);
        if (ok > k) over += ow;
        if (ok == k) same += ow;
      }
      const bool hit = i >= 0 && over < left && left <= over + same;
      const int who = __ffs(__ballot_sync(0xffffffffu, hit)) - 1;
      left -= __shfl_sync(0xffffffffu, over, who);
      return __shfl_sync(0xffffffffu, k, who);
    }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    auto sum_from = [&](unsigned from) {
      unsigned long long some = 0;
      for (int i = lane * q; i < (lane + 1) * q; ++i)
        if (keys[i] >= from && keys[i] <= high) some += MASS ? weight(i) : 1ull;
      return warp_sum(some);
    };
    const unsigned key = largest_key(low, high, left, sum_from);
    if (key < high) left -= sum_from(key + 1);
    return key;
  }
};
// words of a warp's shared memory: keys, 2^t where weights are needed, bins and list where entries may
// be filtered
__host__ __device__ constexpr int short_words(int q, bool mass, bool filters) {
  return q * 32 * (mass ? 2 : 1) + (filters ? 2 * SBINS + 32 : 0);
}

template <class T, bool MASS>
__global__ void __launch_bounds__(SW * 32)
    k_sample_short(int64_t rows, int n, int q, bool filters, const T* __restrict__ logits, int64_t stride,
                   const uint64_t* __restrict__ words, erc_sample_rule rule,
                   int32_t* __restrict__ ids, float* __restrict__ logp,
                   int32_t* __restrict__ kept) {
  extern __shared__ unsigned short_buffer[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned* keys = short_buffer + warp * short_words(q, MASS, filters);
  float* powers = reinterpret_cast<float*>(keys + q * 32);  // MASS only
  unsigned* bins = keys + (MASS ? 2 : 1) * q * 32;
  for (int64_t row = (int64_t)blockIdx.x * SW + warp; row < rows; row += (int64_t)gridDim.x * SW) {
    const T* x = logits + row * stride;
    const RowRule r = row_rule(rule, row);
    float m = -INFINITY;
#pragma unroll 4
    for (int i = lane; i < q * 32; i += 32) {
      const float l = i < n ? clean_score(to_f32(x[i])) : -INFINITY;
      m = fmaxf(m, l);
      keys[i] = __float_as_uint(l);
    }
    m = order_value(__reduce_max_sync(0xffffffffu, order_key(__fadd_rn(m, 0.f))));
    if (m == -INFINITY) {
      if (lane == 0) {
        ids[row] = -1;
        logp[row] = -INFINITY;
        kept[row] = 0;
      }
      __syncwarp();
      continue;
    }
    const ShortRow sr = {keys, powers, bins, bins + 2 * SBINS, q, m, r.scale};
    const float least_t = r.least <= 1 ? -41.5f : log2f((float)r.least - 0.5f) - 40.01f;
    __syncwarp();
    // a lane's own entries
    unsigned* mine = keys + lane * q;
    unsigned long long mass = 0;
    unsigned above = 0;
    for (int i = 0; i < q; ++i) {
      const float l = __uint_as_float(mine[i]);
      const float t = l == -INFINITY ? -INFINITY : below_max(l, m, r.scale);
      unsigned long long w = 0;
      float v = 0.f;
      if (t >= least_t) {
        v = t > -41.5f ? pow2_float(t, -41.f) : 0.f;
        unsigned hi[2], lo[2];
        split_weights(pair(v, v), hi, lo);
        w = join_parts(hi[0], lo[0]);
        if (w < r.least) w = 0;
      }
      mine[i] = w ? order_key(l) : 0u;
      if (MASS) powers[lane * q + i] = v;
      mass += w;
      above += w != 0;
    }
    __syncwarp();
    auto weight_of = [&](unsigned k) {
      return k ? fixed_weight(below_max(order_value(k), m, r.scale)) : 0ull;
    };
    unsigned theta = 0, ties = 0xffffffffu, tied = 0;
    unsigned number = __reduce_add_sync(0xffffffffu, above);
    const bool by_k = r.top_k < number, by_p = MASS && r.part != 0xffffffffu;
    if (by_k) {
      unsigned long long left = r.top_k;
      theta = sr.find<false>(0u, left);
      ties = (unsigned)left;
      number = r.top_k;
    }
    if (by_p) {
      unsigned long long over = mass;
      if (by_k) {
        over = 0;
        for (int i = 0; i < q; ++i)
          if (mine[i] > theta) over += sr.weight(lane * q + i);
      }
      over = warp_sum(over);
      const unsigned long long wt = weight_of(theta);
      const unsigned long long total = over + (by_k ? ties * wt : 0ull);
      unsigned long long target = (total >> 31) * r.part + (((total & 0x7fffffffull) * r.part) >> 31);
      if (!target) target = 1;
      if (over < target) {
        ties = (unsigned)((target - over + wt - 1) / wt);
      } else {
        theta = sr.find<MASS>(theta, target);
        const unsigned long long w = weight_of(theta);
        ties = (unsigned)((target + w - 1) / w);
      }
      number = 0;
      for (int i = 0; i < q; ++i) number += mine[i] > theta;
      number = __reduce_add_sync(0xffffffffu, number) + ties;
    }
    if (by_k || by_p) {
      mass = 0;
      const unsigned long long wt = weight_of(theta);
      for (int i = 0; i < q; ++i) {
        if (mine[i] > theta) mass += MASS ? sr.weight(lane * q + i) : weight_of(mine[i]);
        tied += mine[i] == theta;
      }
      const unsigned earlier = warp_inclusive(tied) - tied;
      tied = earlier < ties ? min(tied, ties - earlier) : 0u;  // of the lane's ties, those kept
      mass += tied * wt;
    }
    const unsigned long long to = warp_inclusive(mass);
    const unsigned long long total = __shfl_sync(0xffffffffu, to, 31);
    const unsigned long long at = __umul64hi(words[row], total);
    const int owner = 31 - __clz(__ballot_sync(0xffffffffu, to - mass <= at && mass));
    unsigned long long before = __shfl_sync(0xffffffffu, to - mass, owner);
    unsigned left = __shfl_sync(0xffffffffu, tied, owner);  // ties of the owner's that are kept
    for (int i0 = 0; i0 < q; i0 += 32) {  // the owner's entries, one a lane
      const unsigned k = i0 + lane < q ? keys[owner * q + i0 + lane] : 0u;
      const bool tie = theta && k == theta;
      const unsigned tie_lanes = __ballot_sync(0xffffffffu, tie);
      const unsigned earlier = __popc(tie_lanes & ((1u << lane) - 1));
      const unsigned long long w = k > theta || (tie && earlier < left) ? weight_of(k) : 0ull;
      const unsigned long long in = before + warp_inclusive(w);
      if (at < in && in - w <= at) {
        const unsigned long long rest = total - w;
        ids[row] = owner * q + i0 + lane;
        kept[row] = (int32_t)number;
        logp[row] = w > rest ? log1pf(-__fdiv_rn(__ull2float_rn(rest), __ull2float_rn(total)))
                             : logf(__fdiv_rn(__ull2float_rn(w), __ull2float_rn(total)));
      }
      left -= min(left, (unsigned)__popc(tie_lanes));
      before = __shfl_sync(0xffffffffu, in, 31);
    }
    __syncwarp();
  }
}

}  // namespace

// enqueues the kernel for scores of type T; each type's kernels are a translation unit
template <class T>
erc_status launch_rows(int64_t rows, int64_t n, const T* logits, int64_t stride,
                       const uint64_t* words, const erc_sample_rule& rule, int32_t* ids,
                       float* logp, int32_t* kept, cudaStream_t s) {
  // a warp a row, but a whole block for few rows (1 x 1000, top-k: 27 us by a warp, 8 by a block)
  if (n <= 256 || (n <= SHORT && rows > 2 * sm_count())) {
    const int q = short_q(n);
    const bool mass = rule.top_p < 1.f || rule.top_p_rows;
    const bool filters = mass || rule.top_k > 0 || rule.top_k_rows || !(rule.temperature > 0.f) ||
                         rule.temperature_rows;
    const size_t bytes = (size_t)SW * short_words(q, mass, filters) * 4;
    auto kernel = mass ? k_sample_short<T, true> : k_sample_short<T, false>;
    // the longest row's, whatever this one's: a limit of its own could undercut another thread's call
    // between its setting and its launch
    constexpr int most = SW * 4 * short_words(short_q(SHORT), true, true);
    if (bytes > 48 * 1024)
      ERC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    const int64_t blocks = (rows + SW - 1) / SW;
    kernel<<<(unsigned)(blocks < 0x7fffffff ? blocks : 0x7fffffff), SW * 32, bytes, s>>>(
        rows, (int)n, q, filters, logits, stride, words, rule, ids, logp, kept);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  }
  // Blocks of 512 threads, two an SM; where the rows give an SM no second block, blocks of 1024 take
  // long parts.  112: seven clusters of 16 such blocks fit the machine at once.
  const int C = blocks_of(rows, n);
  const bool many = C > 1 && rows * C <= 112 && n >= (int64_t)C * 512 * 64;
  static std::atomic<uint64_t> ready{0};  // devices whose kernels have their attributes, one bit each
  int dev = 0;
  ERC_CUDA(cudaGetDevice(&dev));
  if (dev >= 64 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, true, 128>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(128)));
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, true, 512>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(512)));
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, false, 512>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(512)));
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, false, 1024>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(1024)));
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, false, 512>,
                                  cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    ERC_CUDA(cudaFuncSetAttribute(k_sample_rows<T, false, 1024>,
                                  cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows < 65535 ? rows : 65535) * C);
  const bool small = C == 1 && n <= SMALL && rows > sm_count();
  const int threads = small ? 128 : many ? 1024 : 512;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = ring_bytes(threads);
  cfg.stream = s;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = C;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = C > 1;
  auto kernel = small    ? k_sample_rows<T, true, 128>
                : C == 1 ? k_sample_rows<T, true, 512>
                : many ? k_sample_rows<T, false, 1024>
                       : k_sample_rows<T, false, 512>;
  ERC_CUDA(cudaLaunchKernelEx(&cfg, kernel, rows, n, logits, stride, words, rule, C, ids, logp, kept));
  count_launches(1);
  return ERC_OK;
}

}  // namespace erc
