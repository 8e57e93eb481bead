// score_rows.cu -- log probability of a given entry of each row of scores, the row's entropy and its
// best entries, and the scores' gradient.
//
// With c = log2(e) / temperature, m the largest score and t = (l - m) c, T = sum 2^t and u = sum 2^t t
// give ln Z = ln T and the entropy ln T - ln2 u / T.  A part of a row (at most 48 KB) arrives in shared
// memory by one asynchronous copy; a first pass finds its maximum, a second its sums, so an entry costs one
// exponential and no part scales its sums.  Parts join by d = (m_part - m) c: u <- 2^d (u + d T), T <- 2^d T.
// t is kept above -1000, where 2^t is 0, so that no product of 0 and infinity appears.
//
// The best entries need no pass of their own: the first one notes the largest score of each 32 vectors
// (a segment, 512 bytes).  The k segments with the best maxima (ties to the first) hold the k best
// entries: an entry elsewhere is behind the k maxima.  Only these are searched, in shared memory.
//
// Up to 8 parts are a cluster, whose first block joins them through distributed shared memory; more go
// through a workspace and a second kernel.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int ST = 256;          // threads of a block
constexpr int SW = ST / 32;      // its warps
constexpr int SV = 4;            // vectors a thread holds at a time
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

struct Sum {
  float m, T, u;  // m: LOWEST where nothing was met (T = 0)
};
__device__ __forceinline__ void raise(Sum& a, float m, float c) {
  const float d = scaled(a.m, m, c), f = exp2_fast(d);
  a.u = f * fmaf(d, a.T, a.u);
  a.T *= f;
  a.m = m;
}
__device__ __forceinline__ Sum join(Sum a, Sum b, float c) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m, c);
  raise(b, m, c);
  return {m, a.T + b.T, a.u + b.u};
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

// the terms of a vector, with the maximum known
template <class T>
__device__ __forceinline__ void add_vector(Sum& a, uint4 v, float c) {
  float l[ScoreVec<T>::N];
  unpack_scores(v, l, T());
#pragma unroll
  for (int i = 0; i < ScoreVec<T>::N; ++i) {
    const float t = scaled(l[i], a.m, c), e = exp2_fast(t);
    a.T += e;
    a.u = fmaf(e, t, a.u);
  }
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
};

__device__ __forceinline__ float log_p(float l, float m, float lnT, float temperature) {
  return l == -INFINITY ? -INFINITY : (l == m ? 0.f : __fdiv_rn(l - m, temperature)) - lnT;
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
  const bool some = !(a.T <= 0.f);  // NaN: a copy that did not land
  const float lnT = some ? logf(a.T) : -INFINITY, entropy = some ? lnT - LN2 * (a.u / a.T) : 0.f;
  if (o.entropy) o.entropy[row] = entropy < 0.f ? 0.f : entropy;
  if (o.norm) {
    o.norm[2 * row] = some ? a.m : -INFINITY;
    o.norm[2 * row + 1] = lnT;
  }
  if (o.logp) o.logp[row] = g.id < 0 ? 0.f : some ? log_p(g.l, a.m, lnT, o.temperature) : -INFINITY;
}

// an entry of a row's part in the workspace
struct Best {
  unsigned key, id;
};
__device__ __forceinline__ bool ahead(unsigned ka, unsigned ia, unsigned kb, unsigned ib) {
  return ka > kb || (ka == kb && ia < ib);
}

struct TopScratch {
  unsigned seg[MAX_PARTS];  // best key of each segment
  int chosen[KMAX];         // the k best segments, best first
  unsigned least;           // the key of the last of them
  int segments, found;
  Best list[KMAX * KMAX];   // what they hold from `least` on, at most k of each
};

// The k best of the entries behind s.seg[0 .. nseg): fetch(segment, lane, e, keys, ids) gives the
// e-th of a lane's ENTRIES of a segment.  put(rank, key, id) takes the results.
template <int ENTRIES, class Fetch, class Put>
__device__ __forceinline__ void select_top(TopScratch& s, int nseg, int k, Fetch&& fetch, Put&& put) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) s.segments = s.found = 0, s.least = 0;
  __syncthreads();
  for (int i = tid; i < nseg; i += ST) {
    const unsigned mine = s.seg[i];
    if (mine <= MASKED_KEY) continue;
    int before = 0;
    for (int j = 0; j < nseg; ++j) before += ahead(s.seg[j], j, mine, i);
    if (before < k) {
      s.chosen[before] = i;
      atomicMax(&s.segments, before + 1);
      if (before == k - 1) s.least = mine;
    }
  }
  __syncthreads();
  const unsigned least = max(s.least, MASKED_KEY + 1);
  for (int j = warp; j < s.segments; j += SW) {
    unsigned key[ENTRIES], id[ENTRIES];
    int mine = 0;
    fetch(s.chosen[j], lane, key, id);
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
      if (key[i] < least) key[i] = 0;
      mine += key[i] != 0;
    }
    const int all = __reduce_add_sync(0xffffffffu, mine);
    if (all <= k) {
      int at = mine ? atomicAdd(&s.found, mine) : 0;
#pragma unroll
      for (int i = 0; i < ENTRIES; ++i)
        if (key[i]) s.list[at++] = {key[i], id[i]};
    } else {  // many equal ones: the first k of the segment, one after another
      for (int r = 0; r < k; ++r) {
        unsigned bk = 0, bi = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i)
          if (key[i] && ahead(key[i], id[i], bk, bi)) bk = key[i], bi = id[i];
        const unsigned top = __reduce_max_sync(0xffffffffu, bk);
        const unsigned first = __reduce_min_sync(0xffffffffu, bk == top ? bi : 0xffffffffu);
        if (lane == 0) s.list[atomicAdd(&s.found, 1)] = {top, first};
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i)
          if (id[i] == first) key[i] = 0;
      }
    }
  }
  __syncthreads();
  const int found = s.found;
  for (int i = tid; i < found; i += ST) {
    const Best b = s.list[i];
    int before = 0;
    for (int j = 0; j < found; ++j) before += ahead(s.list[j].key, s.list[j].id, b.key, b.id);
    if (before < k) put(before, b.key, b.id);
  }
  for (int r = found + tid; r < k; r += ST) put(r, 0u, 0u);  // fewer than k
}

__device__ __forceinline__ void put_best(const ScoreOut& o, int64_t row, Sum a, float lnT, int rank, unsigned key,
                                         unsigned id) {
  o.top_ids[row * o.k + rank] = key ? (int32_t)id : -1;
  o.top_logp[row * o.k + rank] = key ? log_p(order_value(key), a.m, lnT, o.temperature) : -INFINITY;
}

// the sums of a block whose threads share a maximum, in the order of its warps
__device__ __forceinline__ Sum block_sum(Sum a, Sum* part) {
  a.T = warp_sum(a.T);
  a.u = warp_sum(a.u);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
  __syncthreads();
  Sum all = part[0];
#pragma unroll
  for (int w = 1; w < SW; ++w) all.T += part[w].T, all.u += part[w].u;
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

// waits for a copy into shared memory; false when a second or so was not enough (the row's results are NaN then)
__device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity) {
  for (unsigned i = 0; i < (1u << 22); ++i) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done)
                 : "r"(bar), "r"(parity)
                 : "memory");
    if (done) return true;
  }
  return false;
}

template <class T>
constexpr int part_smem(bool top) { return SEGS * 512 + (top ? (int)sizeof(TopScratch) : 0); }

// A block takes one of the `parts` of a row, `per` vectors each (a multiple of 32).  CLUSTERED: the parts of a row are a
// cluster.  Blocks start with a task and take every gridDim.x-th one.
template <class T, bool TOP, bool CLUSTERED>
__global__ void __launch_bounds__(ST) k_score_part(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                   int parts, int per, ScoreOut o, Sum* __restrict__ sums,
                                                   Best* __restrict__ best) {
  constexpr int N = ScoreVec<T>::N;
  constexpr unsigned NONE = 0xffffffffu;
  __shared__ Sum part[SW];
  __shared__ Sum joined;
  __shared__ float top_of[SW];
  __shared__ Best mine[KMAX];
  __shared__ __align__(8) uint64_t bar_word;
  extern __shared__ __align__(16) char smem[];
  uint4* held = reinterpret_cast<uint4*>(smem);
  TopScratch& top = *reinterpret_cast<TopScratch*>(smem + SEGS * 512);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t bar = shared_at(&bar_word);
  if (tid == 0) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  uint32_t parity = 0;
  const int64_t tasks = rows * parts;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t row = task / parts;
    const int which = (int)(task - row * parts);
    const T* x = logits + row * stride;
    const RowView<T> view(x, n);
    const int first = which * per, count = max(min(per, view.vectors - first), 0);
    // whole vectors arrive by the copy, those that the row shares with its neighbours element by element
    const int lo = min(first == 0 && view.skew ? 1 : 0, count), hi = max(min(first + count, view.whole()) - first, lo);
    if (tid == 0) {
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
    if (tid == 32) {
      for (int v = hi; v < count; ++v) held[v] = view.fetch(first + v);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    Given g = {-1, 0.f};
    if (tid == 0 && (CLUSTERED ? which == 0 : parts == 1)) g = given_of(o, row, x, n);
    bool ok = true;
    if (hi > lo) {
      ok = landed(bar, parity);
      parity ^= 1;
    }
    ok = __syncthreads_and(ok);

    float m = LOWEST;
    for (int v0 = warp * 32; v0 < count; v0 += ST) {
      const int at = v0 + lane;
      const float here = at < count ? max_score(held[at], T()) : -INFINITY;
      if (TOP) {
        const unsigned key = __reduce_max_sync(NONE, order_key(__fadd_rn(here, 0.f)));
        if (lane == 0) top.seg[v0 / 32] = key;
      }
      m = fmaxf(m, here);
    }
    m = warp_max(m);
    if (lane == 0) top_of[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SW; ++w) m = fmaxf(m, top_of[w]);
    Sum a = {m, 0.f, 0.f};
    for (int at = tid; at < count; at += ST) add_vector<T>(a, held[at], o.c);
    a = block_sum(a, part);
    if (!ok) a = {NAN, NAN, NAN};
    if (TOP) {
      const bool alone = !CLUSTERED && parts == 1;
      const float lnT = alone && a.T > 0.f ? logf(a.T) : -INFINITY;
      select_top<N>(
          top, (count + 31) / 32, o.k,
          [&](int seg, int l, unsigned* key, unsigned* id) {
            const int at = seg * 32 + l;
            float s[N];
            uint4 v = make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
            if (at < count) v = held[at];
            unpack_scores(v, s, T());
#pragma unroll
            for (int i = 0; i < N; ++i) {
              key[i] = order_key(__fadd_rn(s[i], 0.f));
              id[i] = (unsigned)((first + at) * N + i - view.skew);
            }
          },
          [&](int rank, unsigned key, unsigned id) {
            if (CLUSTERED)
              mine[rank] = {key, id};
            else if (alone)
              put_best(o, row, a, lnT, rank, key, id);
            else
              best[task * o.k + rank] = {key, id};
          });
    }
    if constexpr (CLUSTERED) {
      if (tid == 0) joined = a;
      cluster_sync_all();
      if (which == 0) {
        Sum all = a;
        for (int p = 1; p < parts; ++p) {
          const uint32_t at = of_block(shared_at(&joined), p);
          const Sum other = {__uint_as_float(peer_word(at)), __uint_as_float(peer_word(at + 4)),
                             __uint_as_float(peer_word(at + 8))};
          all = join(all, other, o.c);
        }
        if (tid == 0) finish_row(o, row, g, all);
        if (TOP) {
          const float lnT = all.T > 0.f ? logf(all.T) : -INFINITY;
          if (tid < parts) top.seg[tid] = peer_word(of_block(shared_at(&mine[0].key), tid));
          __syncthreads();
          select_top<1>(
              top, parts, o.k,
              [&](int p, int l, unsigned* key, unsigned* id) {
                key[0] = id[0] = 0;
                if (l < o.k) {
                  const uint32_t at = of_block(shared_at(&mine[l]), p);
                  key[0] = peer_word(at);
                  id[0] = peer_word(at + 4);
                }
              },
              [&](int rank, unsigned key, unsigned id) { put_best(o, row, all, lnT, rank, key, id); });
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
    Sum a = {LOWEST, 0.f, 0.f};
    for (int p = threadIdx.x; p < parts; p += ST) a = join(a, sums[row * parts + p], o.c);
    const Best* mine = best + row * parts * o.k;
    if (TOP)
      for (int p = threadIdx.x; p < parts; p += ST) top.seg[p] = mine[p * o.k].key;
#pragma unroll
    for (int w = 16; w; w >>= 1) {
      const Sum b = {__shfl_xor_sync(0xffffffffu, a.m, w), __shfl_xor_sync(0xffffffffu, a.T, w),
                     __shfl_xor_sync(0xffffffffu, a.u, w)};
      a = join(a, b, o.c);  // the same on both sides: sums and maxima commute
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int w = 1; w < SW; ++w) a = join(a, part[w], o.c);
    if (threadIdx.x == 0) finish_row(o, row, g, a);
    if (TOP) {
      const float lnT = a.T > 0.f ? logf(a.T) : -INFINITY;
      select_top<1>(
          top, parts, o.k,
          [&](int p, int l, unsigned* key, unsigned* id) {
            const Best b = l < o.k ? mine[p * o.k + l] : Best{0u, 0u};
            key[0] = b.key;
            id[0] = b.id;
          },
          [&](int rank, unsigned key, unsigned id) { put_best(o, row, a, lnT, rank, key, id); });
    }
    __syncthreads();
  }
}

// a warp takes a row of at most 32 VPL vectors
template <class T, int VPL, bool TOP>
__global__ void __launch_bounds__(ST) k_score_short(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                    ScoreOut o) {
  constexpr int N = ScoreVec<T>::N;
  const int lane = threadIdx.x & 31;
  for (int64_t row = ((int64_t)blockIdx.x * ST + threadIdx.x) >> 5; row < rows; row += (int64_t)gridDim.x * SW) {
    const T* x = logits + row * stride;
    const RowView<T> view(x, n);
    uint4 v[VPL];
    float m = LOWEST;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int at = j * 32 + lane;
      if (at < view.vectors)
        v[j] = view.fetch(at);
      else
        v[j] = make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
    }
    Given g = {-1, 0.f};
    if (lane == 0) g = given_of(o, row, x, n);
#pragma unroll
    for (int j = 0; j < VPL; ++j) m = fmaxf(m, max_score(v[j], T()));
    Sum a = {warp_max(m), 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < VPL; ++j) add_vector<T>(a, v[j], o.c);
    a.T = warp_sum(a.T);
    a.u = warp_sum(a.u);
    if (lane == 0) finish_row(o, row, g, a);
    if (TOP) {
      const float lnT = a.T > 0.f ? logf(a.T) : -INFINITY;
      unsigned pk = 0xffffffffu, pi = 0;  // the one found last
      for (int r = 0; r < o.k; ++r) {
        unsigned bk = 0, bi = 0xffffffffu;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
          float s[N];
          unpack_scores(v[j], s, T());
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const unsigned key = order_key(__fadd_rn(s[i], 0.f)), id = (unsigned)((j * 32 + lane) * N + i - view.skew);
            if (key > MASKED_KEY && ahead(pk, pi, key, id) && ahead(key, id, bk, bi)) bk = key, bi = id;
          }
        }
        pk = __reduce_max_sync(0xffffffffu, bk);
        pi = __reduce_min_sync(0xffffffffu, bk == pk ? bi : 0xffffffffu);
        if (lane == 0) put_best(o, row, a, lnT, r, pk, pi);
        if (pk == 0) {
          for (int q = r + 1 + lane; q < o.k; q += 32) put_best(o, row, a, lnT, q, 0u, 0u);
          break;
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
struct RowGrad {
  float m, lnZ, shift, g, gh, H, inv;
  int id;
  __device__ __forceinline__ float operator()(float l, int i, float c) const {
    if (l == -INFINITY) return 0.f;
    const float t = scaled(l, m, c), lp = fmaf(t, LN2, -lnZ);
    const float p = exp2_fast(t - shift);
    float v = -p * fmaf(gh, lp + H, g);
    if (i == id) v += g;
    return v * inv;
  }
};

template <class T>
__global__ void __launch_bounds__(ST) k_score_backward(int64_t rows, int64_t n, const T* __restrict__ logits,
                                                       int64_t stride, int parts, ScoreGrad o, T* __restrict__ dlogits) {
  constexpr int N = ScoreVec<T>::N;
  const int64_t tasks = rows * parts;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t row = task / parts;
    const int which = (int)(task - row * parts);
    const T* x = logits + row * stride;
    T* out = dlogits + row * n;
    const RowView<T> view(x, n);
    RowGrad r;
    r.m = o.norm[2 * row];
    r.lnZ = o.norm[2 * row + 1];
    r.shift = r.lnZ * LOG2E;
    r.id = o.ids ? o.ids[row] : -1;
    r.g = o.dlogp && r.id >= 0 && r.id < n && clean_score(to_f32(x[r.id])) != -INFINITY ? o.dlogp[row] : 0.f;
    r.gh = o.dentropy ? o.dentropy[row] : 0.f;
    r.H = o.dentropy ? o.entropy[row] : 0.f;
    r.inv = __frcp_rn(o.temperature);
    const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    T* shifted = out - view.skew;
    for (int v0 = which * ST * SV; v0 < view.vectors; v0 += parts * ST * SV) {
      uint4 v[SV];
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        const int at = v0 + j * ST + threadIdx.x;
        if (at < view.vectors) v[j] = view.fetch(at);
      }
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        const int at = v0 + j * ST + threadIdx.x;
        if (at >= view.vectors) continue;
        float l[N];
        unpack_scores(v[j], l, T());
        union Piece {
          uint4 raw;
          T t[N];
          __device__ Piece() {}
        } q;
        const int e = at * N - view.skew;
#pragma unroll
        for (int i = 0; i < N; ++i) q.t[i] = from_f32<T>(r(l[i], e + i, o.c));
        if (same && e >= 0 && e + N <= n) {
          reinterpret_cast<uint4*>(shifted)[at] = q.raw;
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
  const int64_t wanted = ((int64_t)sm_count() * 4 + rows - 1) / rows;
  const int64_t most = (segments + 2 * SW - 1) / (2 * SW);  // two vectors a thread at least
  int64_t parts = wanted < most ? wanted : most;
  if (parts < least) parts = least;
  if (parts > CLUSTER && least <= CLUSTER && (rows * CLUSTER >= 2 * sm_count() || parts <= 3 * CLUSTER)) parts = CLUSTER;
  if (parts > MAX_PARTS) parts = MAX_PARTS;
  const int64_t each = (segments + parts - 1) / parts;
  return {(int)((segments + each - 1) / each), (int)each * 32};
}
bool short_rows(int64_t n, int32_t type) { return n / (16 / type_bytes(type)) + 2 <= 256; }

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
  if (sp.parts <= CLUSTER) return 0;
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
  const ScoreOut o = {ids, logp, entropy, norm, top_ids, top_logp, temperature, LOG2E / temperature, k};
  const cudaStream_t s = as_stream(stream);
  const bool brief = short_rows(n, type);
  const Split sp = brief ? Split{1, 0} : split_rows(rows, n, type);
  ScorePlan p = {};
  if (sp.parts > CLUSTER) {
    if (!ws || ws_bytes < erc_score_rows_workspace_size(rows, n, type, k))
      return set_error(ERC_ERR_CAPACITY, "workspace too small");
    Arena ar(reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~uintptr_t(255)));
    plan_scores(ar, p, rows, sp.parts, k);
  }
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const T* x = static_cast<const T*>(logits);
    if (brief) {
      const int64_t vectors = n / ScoreVec<T>::N + 2, blocks = (rows + SW - 1) / SW, most = (int64_t)sm_count() * 64;
      const unsigned grid = (unsigned)(blocks < most ? blocks : most);
      auto launch = [&](auto vpl) {
        constexpr int V = decltype(vpl)::value;
        (k ? k_score_short<T, V, true> : k_score_short<T, V, false>)<<<grid, ST, 0, s>>>(rows, n, x, stride, o);
      };
      if (vectors <= 32)
        launch(ic<1>());
      else if (vectors <= 64)
        launch(ic<2>());
      else if (vectors <= 128)
        launch(ic<4>());
      else
        launch(ic<8>());
      count_launches(1);
    } else {
      const int smem = part_smem<T>(k > 0);
      const int64_t tasks = rows * sp.parts;
      const bool together = sp.parts > 1 && sp.parts <= CLUSTER;
      auto kernel = together ? (k ? k_score_part<T, true, true> : k_score_part<T, false, true>)
                             : (k ? k_score_part<T, true, false> : k_score_part<T, false, false>);
      ERC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
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
    const int64_t vectors = n / ScoreVec<T>::N + 2, steps = (vectors + ST * SV - 1) / (ST * SV);
    const int64_t wanted = ((int64_t)sm_count() * 8 + rows - 1) / rows;
    const int parts = (int)(steps < wanted ? steps : wanted);
    const int64_t tasks = rows * parts, most = (int64_t)sm_count() * 64;
    k_score_backward<T><<<(unsigned)(tasks < most ? tasks : most), ST, 0, as_stream(stream)>>>(
        rows, n, static_cast<const T*>(logits), stride, parts, o, static_cast<T*>(dlogits));
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
    return ERC_OK;
  });
}
