// score_rows.cu -- log probability of a given entry of each row of scores, the row's entropy and its
// best entries, and the scores' gradient.
//
// One pass: with c = log2(e) / temperature, m the largest score so far, t = (l - m) c and e = 2^t, a
// thread keeps T = sum e and u = sum e t.  A new maximum scales both: with d = (m_old - m_new) c,
// u <- 2^d (u + d T), T <- 2^d T.  Then ln Z = ln T and the entropy is ln T - ln2 u / T.  t is kept
// above -1000, where 2^t is 0, so that no product of 0 and infinity appears.
//
// The best entries need no second pass either: every warp notes the largest score of each 32 vectors
// (a segment, 512 bytes).  The k segments with the best maxima (ties to the first) hold the k best
// entries: an entry elsewhere is behind the k maxima.  Only these segments are read again.
#include "choice.cuh"

namespace erc {
namespace {

constexpr int ST = 256;          // threads of a block
constexpr int SW = ST / 32;      // its warps
constexpr int SV = 4;            // vectors a thread holds at a time
constexpr int SEGS = 256;        // segments of a block's part of a row, at most
constexpr int MAX_PARTS = 512;   // parts of a row, at most
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
__device__ __forceinline__ Sum lane_join(Sum a, float c, int width) {
  for (int o = width / 2; o; o >>= 1) {
    const Sum b = {__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.T, o),
                   __shfl_xor_sync(0xffffffffu, a.u, o)};
    a = join(a, b, c);  // the same on both sides: sums and maxima commute
  }
  return a;
}

// `count` vectors of a thread: first their maximum, then their terms
template <class T, int COUNT>
__device__ __forceinline__ void add_vectors(Sum& a, const uint4* v, float m, float c) {
  if (m > a.m) raise(a, m, c);
#pragma unroll
  for (int j = 0; j < COUNT; ++j) {
    float l[ScoreVec<T>::N];
    unpack_scores(v[j], l, T());
#pragma unroll
    for (int i = 0; i < ScoreVec<T>::N; ++i) {
      const float t = scaled(l[i], a.m, c), e = exp2_fast(t);
      a.T += e;
      a.u = fmaf(e, t, a.u);
    }
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

template <class T>
__device__ __forceinline__ void finish_row(const ScoreOut& o, int64_t row, const T* x, int64_t n, Sum a) {
  const bool some = a.T > 0.f;
  const float lnT = some ? logf(a.T) : -INFINITY;
  if (o.entropy) o.entropy[row] = some ? fmaxf(lnT - LN2 * (a.u / a.T), 0.f) : 0.f;
  if (o.norm) {
    o.norm[2 * row] = some ? a.m : -INFINITY;
    o.norm[2 * row + 1] = lnT;
  }
  if (o.logp) {
    const int32_t id = o.ids[row];
    float p = 0.f;
    if (id >= 0 && id < n) p = some ? log_p(clean_score(to_f32(x[id])), a.m, lnT, o.temperature) : -INFINITY;
    o.logp[row] = p;
  }
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

__device__ __forceinline__ Sum block_join(Sum a, float c, Sum* part) {
  a = lane_join(a, c, 32);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
  __syncthreads();
  Sum all = part[0];
#pragma unroll
  for (int w = 1; w < SW; ++w) all = join(all, part[w], c);
  return all;
}

// a block takes one of the `parts` of a row, `per` vectors each (a multiple of 32)
template <class T, bool TOP>
__global__ void __launch_bounds__(ST) k_score_part(int64_t rows, int64_t n, const T* __restrict__ logits, int64_t stride,
                                                   int parts, int per, ScoreOut o, Sum* __restrict__ sums,
                                                   Best* __restrict__ best) {
  constexpr int N = ScoreVec<T>::N;
  __shared__ Sum part[SW];
  extern __shared__ __align__(16) char smem[];
  TopScratch& top = *reinterpret_cast<TopScratch*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t tasks = rows * parts;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t row = task / parts;
    const int which = (int)(task - row * parts);
    const T* x = logits + row * stride;
    const RowView<T> view(x, n);
    const int first = which * per, last = min(first + per, view.vectors);
    Sum a = {LOWEST, 0.f, 0.f};
    for (int v0 = first; v0 < last; v0 += ST * SV) {
      uint4 v[SV];
      float m = LOWEST;
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        const int at = v0 + j * ST + tid;
        if (at < last)
          v[j] = view.fetch(at);
        else
          v[j] = make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
      }
#pragma unroll
      for (int j = 0; j < SV; ++j) {
        const float here = max_score(v[j], T());
        if (TOP) {
          const unsigned key = __reduce_max_sync(0xffffffffu, order_key(__fadd_rn(here, 0.f)));
          const int seg = (v0 - first + j * ST) / 32 + warp;
          if (lane == 0 && seg * 32 < last - first) top.seg[seg] = key;
        }
        m = fmaxf(m, here);
      }
      add_vectors<T, SV>(a, v, m, o.c);
    }
    a = block_join(a, o.c, part);
    if (parts == 1) {
      if (tid == 0) finish_row(o, row, x, n, a);
    } else if (tid == 0) {
      sums[task] = a;
    }
    if (TOP) {
      const float lnT = parts == 1 && a.T > 0.f ? logf(a.T) : -INFINITY;
      const int nseg = last > first ? (last - first + 31) / 32 : 0;
      select_top<N>(
          top, nseg, o.k,
          [&](int seg, int l, unsigned* key, unsigned* id) {
            const int at = first + seg * 32 + l;
            float s[N];
            uint4 v = make_uint4(masked_word<T>(), masked_word<T>(), masked_word<T>(), masked_word<T>());
            if (at < last) v = view.fetch(at);
            unpack_scores(v, s, T());
#pragma unroll
            for (int i = 0; i < N; ++i) {
              key[i] = order_key(__fadd_rn(s[i], 0.f));
              id[i] = (unsigned)(at * N + i - view.skew);
            }
          },
          [&](int rank, unsigned key, unsigned id) {
            if (parts == 1)
              put_best(o, row, a, lnT, rank, key, id);
            else
              best[task * o.k + rank] = {key, id};
          });
    }
    __syncthreads();
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
    Sum a = {LOWEST, 0.f, 0.f};
    for (int p = threadIdx.x; p < parts; p += ST) a = join(a, sums[row * parts + p], o.c);
    a = block_join(a, o.c, part);
    if (threadIdx.x == 0) finish_row(o, row, logits + row * stride, n, a);
    if (TOP) {
      const float lnT = a.T > 0.f ? logf(a.T) : -INFINITY;
      const Best* mine = best + row * parts * o.k;
      for (int p = threadIdx.x; p < parts; p += ST) top.seg[p] = mine[p * o.k].key;
      __syncthreads();
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
#pragma unroll
    for (int j = 0; j < VPL; ++j) m = fmaxf(m, max_score(v[j], T()));
    Sum a = {LOWEST, 0.f, 0.f};
    add_vectors<T, VPL>(a, v, m, o.c);
    a = lane_join(a, o.c, 32);
    if (lane == 0) finish_row(o, row, x, n, a);
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

// parts of a row: a part is at most SEGS segments, and few rows are split over the whole machine
struct Split {
  int parts, per;  // per: vectors of a part, a multiple of 32
};
Split split_rows(int64_t rows, int64_t n, int32_t type) {
  const int N = 16 / type_bytes(type);
  const int64_t vectors = n / N + 2;  // a row that starts inside a vector ends in one more
  const int64_t segments = (vectors + 31) / 32;
  int64_t parts = (segments + SEGS - 1) / SEGS;
  const int64_t wanted = ((int64_t)sm_count() * 4 + rows - 1) / rows;
  const int64_t most = (segments + 4 * SW - 1) / (4 * SW);  // four vectors a thread at least
  if (parts < wanted) parts = wanted < most ? wanted : most;
  if (parts > MAX_PARTS) parts = MAX_PARTS;
  if (parts < 1) parts = 1;
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
  if (sp.parts == 1) return 0;
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
  if (sp.parts > 1) {
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
      const int64_t tasks = rows * sp.parts, most = (int64_t)sm_count() * 64;
      const unsigned grid = (unsigned)(tasks < most ? tasks : most);
      const size_t smem = k ? sizeof(TopScratch) : 0;
      (k ? k_score_part<T, true> : k_score_part<T, false>)<<<grid, ST, smem, s>>>(rows, n, x, stride, sp.parts, sp.per, o,
                                                                                  p.sums, p.best);
      count_launches(1);
      if (sp.parts > 1) {
        const unsigned joins = (unsigned)(rows < most ? rows : most);
        (k ? k_score_join<T, true> : k_score_join<T, false>)<<<joins, ST, smem, s>>>(rows, n, x, stride, sp.parts, o,
                                                                                     p.sums, p.best);
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
