// expert_ffn_tc.cuh -- the block's products on the tensor cores (tcgen05), bfloat16 and float16.
//
// Every product is D(m, n) = sum_k A(m, k) B(n, k) with m the index that is contiguous in the result, so
// that a warp, whose lanes hold neighbouring m, writes whole sectors:
//
//   product   m       n      k      A                            B
//   IN        gate/up slot   width  w_in, rows of width          x, rows of width
//   OUT       width   slot   inner  w_out, rows of inner         h
//   DH        inner   slot   width  w_out, columns               dy
//   DX        width   slot   2 inner  w_in, columns              (da, db)
//   DWIN      width   2 inner  slot x, columns                   (da, db), columns
//   DWOUT     inner   width  slot   h, columns                   dy, columns
//
// A pair of blocks (a cluster of two) takes a tile of 256 x N, N <= 256: each block holds half of A and
// half of B in shared memory and accumulates its 128 rows of m, one a lane, in tensor memory; the first
// block's thread issues the products of both.  Slots are n, so that a tile at the end of an expert's rows
// costs N = 32, 64, .. columns and not 256, and rows of another expert never mix.  In IN gates and
// factors of the same 8 features alternate in m (the copy's box does that), so that a lane and the lane 8
// further hold a and b of one feature.
//
// Persistent blocks of 20 warps: copies (TMA), products, a warp that zeroes what weight gradients' last copies
// bring of other experts, one that zeroes the rows behind the last expert's, and 16 that read tensor memory and
// write results while the next tile runs in its other half.
//
// Why this tile: a stage of 64 k brings a block 32 KB for 512 clocks of products, and an SM takes in about 64 bytes a
// clock, so 256 x 256 a pair is where copies and products balance; with three quarters of the products left out 8192 x
// 2048 x 4096 still took 0.77 of its time.  Two accumulators fill tensor memory.  What it reaches (8192 slots, one expert,
// 2048 x 4096 bf16): IN 147 us, 1870 TFLOP/s (0.99 of the measured burst rate); OUT 92 us, 1490, 256 tiles on 76
// pairs being 3.4 rounds.  Experts of a few hundred slots (64 x 512 slots of 1024 x 512: IN 52 to 57 us, OUT 36 to 41) saturate
// nothing: tensor pipe 0.57, copies into the SMs 0.56 of 64 bytes a clock, memory 0.63 of the copy rate; their 7 rounds of 16
// stages of 512 clocks are 30 us.  Where the rest goes is not known.  DH also reads (a, b) and writes (da, db) and h, 0.9 GB
// for 80000 slots of 1024: 187 to 190 us, 4.9 TB/s.
//
// What was tried and did not pay: asking for DH's rows ahead (prefetches into L2: 215 -> 240 us, by bulk requests 345;
// reading two or three steps ahead: no change); passing what DH reads and writes through shared memory by tensor copies,
// with 4 stages instead of 6 (200 -> 191 us at a depth of 512, 108 -> 117 at 2048); 8 result warps instead of 16 (DH 209 instead of 200); passing every
// stage on through a warp of each block (the same).  Releases at cluster scope on the way cost a microsecond a stage.
// A wait's look names how long it may sleep (8192 x 2048 x 4096 f16: IN 186 -> 177 us, OUT 106 -> 97 against looks that do not).
//
// Every wait on a barrier ends: after TC_WAIT, or a given number of looks, it gives up.  The block's other roles then
// stop at their next wait; once all have, products and copies in flight are waited for (with limits), tensor memory
// is freed and the status is ERC_ERR_TIMEOUT.  Products may still read, and copies still write, what either block of a
// pair holds: the two end together, and where the products' thread gave up, the results of that tile wait in vain in
// both, so that both pause.  Where it did not, every copy has landed.  Results that were not reached are NaN.
#pragma once

#include <cuda.h>

#include "expert_ffn.cuh"

namespace erc {

constexpr int TC_STAGES = 6;
constexpr int TC_K = 64;                    // depth of a stage: 128 bytes, one row of the swizzle
constexpr int TC_HALF = 128;                // rows of A and of B that a block holds
constexpr int TC_OPERAND = TC_HALF * TC_K * 2;
constexpr int TC_STAGE = 2 * TC_OPERAND;
constexpr int TC_SMEM = TC_STAGES * TC_STAGE + 1024;
constexpr int TC_EPILOGUE = 16;             // warps that write results: a quarter of the rows and of the columns each
constexpr int TC_PART = 256 / (TC_EPILOGUE / 4);
constexpr int TC_THREADS = 128 + 32 * TC_EPILOGUE;
constexpr int tc_cols(int which) { return which == FFN_DH ? 8 : 16; }  // columns that a lane holds at a time
constexpr uint64_t TC_WAIT = 20000000000ull;   // nanoseconds: the sum over the slots of one expert is a tile's longest wait
constexpr uint64_t TC_COPIES = 2000000ull;     // far longer than copies take that are in flight

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t peer_address(uint32_t local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// a look at a barrier, which may sleep for up to `nap` nanoseconds
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity, uint32_t nap) {
  uint32_t done;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(nap)
      : "memory");
  return done;
}
__device__ __forceinline__ uint64_t nanoseconds() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// looks at a barrier `polls` times and for `limit` nanoseconds at most; the clock is read every 256 looks
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity, TcPatience w, uint64_t limit, volatile int* failed) {
  uint64_t start = 0;
  for (unsigned i = 1;; ++i) {
    if (bar_try(bar, parity, w.nap)) return true;
    if ((failed && *failed) || i >= w.polls) return false;
    if (i % 256 == 0) {
      const uint64_t now = nanoseconds();
      if (start == 0) start = now;
      if (now - start > limit) return false;
    }
  }
}
// false when the wait ran out, here or in another role of the block
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* failed, TcPatience w) {
  if (bar_poll(bar, parity, w, TC_WAIT, failed)) return true;
  *failed = 1;
  return false;
}

// A box into this block's shared memory.  PAIR: `bar` is of either block of the pair (a cluster address), else of this one.
template <bool PAIR>
__device__ __forceinline__ void copy_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
        "[%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
            dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
__device__ __forceinline__ void copy_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], "
      "[%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void copy_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int a, int b, int c, int d, int e) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, "
      "%6, %7}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e)
      : "memory");
}

// Shared-memory descriptor of an operand in 128-byte swizzle, 1024-byte aligned atoms.  K contiguous: 8 rows of 128
// bytes an atom, atoms 1024 bytes apart.  M or N contiguous: 64 of them by 8 k an atom, 1024 bytes to the next 8 k and
// 8192 (a box of the copy) to the next 64.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool k_contiguous) {
  uint64_t d = (uint64_t)((addr & 0x3ffff) >> 4);
  d |= (uint64_t)(k_contiguous ? 1 : 8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
      "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
// arrives at the barrier of this offset in both blocks once the products issued so far are done
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"((uint16_t)3)
      : "memory");
}
template <int COLS>
__device__ __forceinline__ void read_tmem(uint32_t addr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  if constexpr (COLS == 8)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
  else
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void read_tmem_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

template <class T>
struct Half2 {
  static constexpr uint32_t FORMAT = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;  // of an operand, in the instruction
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_pair(a, b, T()); }
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return unpack_pair(v, T()); }
};

// a tile: rows of m from m0 on (of both blocks), n columns from n0 on of which `valid` are written, k blocks
struct TcTile {
  int expert, m0, n, valid, blocks, split;
  int64_t n0;       // slot, or row of a weight gradient
  int64_t k0, k1;   // slots of a weight gradient
};

// the experts' slots, the slots of a tile (an expert's tiles are of one size, the last perhaps smaller), and the tiles before
// each expert, in shared memory
struct TcRanges {
  int lo[ERC_ROUTE_MAX_EXPERTS], hi[ERC_ROUTE_MAX_EXPERTS];
  short wide[ERC_ROUTE_MAX_EXPERTS];
  int prefix[ERC_ROUTE_MAX_EXPERTS + 1];
};

// which tiles a product has
template <int WHICH>
struct TcTiles {
  static constexpr bool SLOTS = WHICH <= FFN_DX;
  int m_tiles, n_tiles, depth;  // n_tiles: of a weight gradient
  int n_total, wide, splits;    // a weight gradient's n, its columns a tile, parts of its slots
  __device__ __forceinline__ void init(int D, int F, int splits_) {
    splits = splits_;
    const int m = WHICH == FFN_IN ? 2 * F : WHICH == FFN_DH || WHICH == FFN_DWOUT ? F : D;
    m_tiles = (m + 255) / 256;
    depth = WHICH == FFN_IN || WHICH == FFN_DH ? D : WHICH == FFN_OUT ? F : 2 * F;
    n_total = WHICH == FFN_DWIN ? 2 * F : D;
    wide = n_total <= 128 ? 128 : 256;
    n_tiles = (n_total + wide - 1) / wide;
  }
  __device__ __forceinline__ TcTile at(int t, const TcRanges& of, int experts) const {
    TcTile r;
    if (SLOTS) {
      const int block = t / m_tiles;
      r.m0 = (t - block * m_tiles) * 256;
      int lo = 0, hi = experts;  // the last expert with prefix[e] <= block
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (of.prefix[mid] <= block) lo = mid; else hi = mid;
      }
      r.expert = lo;
      const int wide = of.wide[lo];
      r.n0 = of.lo[lo] + (int64_t)(block - of.prefix[lo]) * wide;
      r.valid = min(of.hi[lo] - (int)r.n0, wide);
      r.n = (r.valid + 31) & ~31;  // a pair's products take multiples of 32
      r.k0 = r.k1 = 0;
      r.blocks = (depth + TC_K - 1) / TC_K;
    } else {
      const int each = m_tiles * n_tiles, of_split = t / each;
      r.expert = of_split / splits;
      r.split = of_split - r.expert * splits;
      const int rest = t - of_split * each;
      r.m0 = rest % m_tiles * 256;
      r.n0 = rest / m_tiles * wide;
      r.n = wide;
      r.valid = min(n_total - (int)r.n0, wide);
      const SlotRange s = split_range({of.lo[r.expert], of.hi[r.expert]}, r.split, splits);
      r.k0 = s.lo;
      r.k1 = s.hi;
      r.blocks = (int)((r.k1 - r.k0 + TC_K - 1) / TC_K);
    }
    return r;
  }
};

// A lane holds row m of two columns, rounded and packed; its neighbour holds m + 1 or m - 1.  They swap: even lanes get
// rows m, m + 1 of the first column, odd lanes rows m - 1, m of the second.
__device__ __forceinline__ uint32_t pair_up(uint32_t own, uint32_t pick) {
  const uint32_t other = __shfl_xor_sync(0xffffffffu, own, 1);
  return __byte_perm(own, other, pick);
}
__device__ __forceinline__ uint32_t pair_pick(int lane) { return lane & 1 ? 0x3276u : 0x5410u; }

// two activations, and their slopes, with the packed instructions: what act_both computes, for arguments that are finite
template <int ACT>
__device__ __forceinline__ void act_pair(uint64_t a, uint64_t& value, uint64_t& slope) {
  float a0, a1, x0, x1;
  unpair(a, a0, a1);
  const uint64_t one = pair(1.f, 1.f), minus = 0x8000000080000000ull;
  if constexpr (ACT == ERC_ACT_SILU) {
    unpair(mul2(a, pair(-LOG2E, -LOG2E)), x0, x1);
    unpair(add2(pair(exp2_hw(x0), exp2_hw(x1)), one), x0, x1);
    const uint64_t q = pair(recip_hw(x0), recip_hw(x1));
    value = mul2(a, q);
    slope = fma2(value, add2(one, q ^ minus), q);
  } else if constexpr (ACT == ERC_ACT_GELU) {
    unpair(fma2(pair(TAIL_STEP, TAIL_STEP), a & 0x7fffffff7fffffffull, one), x0, x1);
    const uint64_t t = pair(recip_hw(x0), recip_hw(x1));
    uint64_t g = pair(tail_coef(8), tail_coef(8));
#pragma unroll
    for (int i = 7; i >= 0; --i) g = fma2(g, t, pair(tail_coef(i), tail_coef(i)));
    unpair(mul2(mul2(a, a), pair(-HALF_LOG2E, -HALF_LOG2E)), x0, x1);
    const uint64_t e = pair(exp2_hw(x0), exp2_hw(x1)), q = mul2(mul2(g, t), e);
    float q0, q1, r0, r1;
    unpair(q, q0, q1);
    unpair(add2(one, q ^ minus), r0, r1);
    const uint64_t below = pair(a0 < 0.f ? q0 : r0, a1 < 0.f ? q1 : r1);
    value = mul2(a, below);
    slope = fma2(mul2(a, e), pair(0.3989422804014327f, 0.3989422804014327f), below);
  } else {
    value = pair(a0 > 0.f || a0 != a0 ? a0 : 0.f, a1 > 0.f || a1 != a1 ? a1 : 0.f);
    slope = pair(a0 > 0.f ? 1.f : 0.f, a1 > 0.f ? 1.f : 0.f);
  }
}

// DH: the pairs (a, a') and (b, b') of the columns that a lane needs, read while the columns before them are at work
constexpr int PRE_PAIRS = tc_cols(FFN_DH) / 2;
struct PrePairs {
  uint32_t a[PRE_PAIRS], b[PRE_PAIRS];
};
// `at`: the lane's byte offset of its first column's row; `two`: bytes of two rows; columns from `live` on are not read
__device__ __forceinline__ void read_pre(const char* a, const char* b, uint32_t at, uint32_t two, int c, int live, PrePairs& r) {
#pragma unroll
  for (int j = 0; j < PRE_PAIRS; ++j) {
    r.a[j] = r.b[j] = 0;
    if (c + 2 * j < live) {
      r.a[j] = __ldg(reinterpret_cast<const uint32_t*>(a + at));
      r.b[j] = __ldg(reinterpret_cast<const uint32_t*>(b + at));
    }
    at += two;
  }
}

// where a lane's results of a tile go: byte offsets from the tile's first row, which 32 bits hold (256 rows of at most
// 2^18 bytes), and the first column that is not its to write
struct TcOut {
  char *first, *second, *third;  // IN: h, gates, factors; DH: (da), (db), h; else the result
  const char *pre_a, *pre_b;
  uint32_t at, at_h, two, two_h;  // offsets of the lane's first column, and of two columns; _h: in rows of inner
  int live, col;                  // col: the lane's column of each pair (IN: of each four)
  bool partial;                   // float32 sums of a part of the slots, one lane a row
};
template <class T, int WHICH>
__device__ __forceinline__ TcOut tile_out(const FfnArgs<T>& p, const TcTile& t, int m_block, int lane, int quad) {
  const int64_t D = p.width, F = p.inner;
  const int odd = lane & 1;
  TcOut o;
  o.partial = false;
  if constexpr (WHICH == FFN_IN) {
    const int f = (t.m0 + m_block) / 2 + quad * 16 + (lane >> 4) * 8 + (lane & 7);
    o.col = 2 * odd + ((lane >> 3) & 1);
    o.live = f < F ? t.valid : 0;
    o.first = reinterpret_cast<char*>(p.h + t.n0 * F + f - odd);
    o.second = reinterpret_cast<char*>(p.pre + t.n0 * 2 * F + f - odd);
    o.third = o.second + F * sizeof(T);
    o.two = 4 * (uint32_t)F * sizeof(T);
    o.two_h = 2 * (uint32_t)F * sizeof(T);
  } else {
    const int m = t.m0 + m_block + quad * 32 + lane;
    const int64_t ld = WHICH == FFN_DH || WHICH == FFN_DWOUT ? F : D;
    o.col = odd;
    o.live = m < ld ? t.valid : 0;
    if constexpr (WHICH == FFN_DH) {
      const int64_t row = t.n0 * 2 * F + m - odd;
      o.first = reinterpret_cast<char*>(p.dpre + row);
      o.second = o.first + F * sizeof(T);
      o.third = reinterpret_cast<char*>(p.h + t.n0 * F + m - odd);
      o.pre_a = reinterpret_cast<const char*>(p.pre_in + row);
      o.pre_b = o.pre_a + F * sizeof(T);
      o.two = 4 * (uint32_t)F * sizeof(T);
      o.two_h = 2 * (uint32_t)F * sizeof(T);
    } else {
      if (WHICH >= FFN_DWIN && p.splits > 1) {
        const int64_t rows = WHICH == FFN_DWIN ? 2 * F : D;
        o.partial = true;
        o.col = 0;
        o.first = reinterpret_cast<char*>(p.partial + (((int64_t)t.split * p.experts + t.expert) * rows + t.n0) * ld + m);
        o.two = o.two_h = 2 * (uint32_t)ld * sizeof(float);
        o.at = o.at_h = 0;
        return o;
      }
      T* out = WHICH == FFN_OUT ? p.y : WHICH == FFN_DX ? p.dx : WHICH == FFN_DWIN ? p.dw_in : p.dw_out;
      if constexpr (WHICH == FFN_DWIN) out += (int64_t)t.expert * 2 * F * D;
      if constexpr (WHICH == FFN_DWOUT) out += (int64_t)t.expert * D * F;
      o.first = reinterpret_cast<char*>(out + t.n0 * ld + m - odd);
      o.two = o.two_h = 2 * (uint32_t)ld * sizeof(T);
    }
  }
  o.at = o.two / 2 * (uint32_t)o.col;
  o.at_h = o.two_h / 2 * (uint32_t)o.col;
  return o;
}

// a lane's columns of a tile from column c on
template <class T, int WHICH, int ACT>
__device__ __forceinline__ void write_columns(const TcOut& o, const float* v, const PrePairs& pre, int c, int lane, bool keep) {
  using H = Half2<T>;
  constexpr int COLS = tc_cols(WHICH);
  const uint32_t pick = pair_pick(lane);
  const int live = o.live - o.col;
  uint32_t at = o.at + (uint32_t)c / 2 * o.two, at_h = o.at_h + (uint32_t)c / 2 * o.two_h;
  if constexpr (WHICH == FFN_IN) {
    // gates where bit 3 of the lane is clear, factors of the same features 8 lanes further: of columns j and j + 1 the
    // gates' lanes keep the first, the factors' lanes the second
    const bool up = lane & 8;
#pragma unroll
    for (int j = 0; j < COLS; j += 4) {
      float g[2], u[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float a = v[j + 2 * q], b = v[j + 2 * q + 1];
        const float got = __shfl_xor_sync(0xffffffffu, up ? a : b, 8);
        g[q] = up ? got : a;
        u[q] = up ? b : got;
      }
      float h0, h1;
      uint64_t value, slope;
      act_pair<ACT>(pair(g[0], g[1]), value, slope);
      unpair(mul2(value, pair(u[0], u[1])), h0, h1);
      const uint32_t h = pair_up(H::pack(h0, h1), pick);
      const bool mine = c + j < live;
      if (mine) *reinterpret_cast<uint32_t*>(o.first + at_h) = h;
      if (keep) {
        const uint32_t gg = pair_up(H::pack(g[0], g[1]), pick), uu = pair_up(H::pack(u[0], u[1]), pick);
        if (mine) {
          *reinterpret_cast<uint32_t*>(o.second + at) = gg;
          *reinterpret_cast<uint32_t*>(o.third + at) = uu;
        }
      }
      at += 2 * o.two;
      at_h += 2 * o.two_h;
    }
  } else if (WHICH >= FFN_DWIN && o.partial) {
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      if (c + j < live) *reinterpret_cast<float*>(o.first + at) = v[j];
      at += o.two / 2;
    }
  } else {
#pragma unroll
    for (int j = 0; j < COLS; j += 2) {
      const bool mine = c + j < live;
      if constexpr (WHICH == FFN_DH) {
        const bool odd = lane & 1;
        const float got = __shfl_xor_sync(0xffffffffu, odd ? v[j] : v[j + 1], 1);
        const uint64_t dh = pair(odd ? got : v[j], odd ? v[j + 1] : got);
        const float2 a = H::unpack(pre.a[j / 2]), b = H::unpack(pre.b[j / 2]);
        const uint64_t bb = pair(b.x, b.y);
        uint64_t value, slope;
        act_pair<ACT>(pair(a.x, a.y), value, slope);
        float x0, x1, y0, y1, z0, z1;
        unpair(mul2(mul2(dh, bb), slope), x0, x1);
        unpair(mul2(dh, value), y0, y1);
        unpair(mul2(value, bb), z0, z1);
        if (mine) {
          *reinterpret_cast<uint32_t*>(o.first + at) = H::pack(x0, x1);
          *reinterpret_cast<uint32_t*>(o.second + at) = H::pack(y0, y1);
          *reinterpret_cast<uint32_t*>(o.third + at_h) = H::pack(z0, z1);
        }
      } else {
        const uint32_t w = pair_up(H::pack(v[j], v[j + 1]), pick);
        if (mine) *reinterpret_cast<uint32_t*>(o.first + at) = w;
      }
      at += o.two;
      at_h += o.two_h;
    }
  }
}

template <class T, int WHICH, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(TC_THREADS, 1)
    k_ffn_tc(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const FfnArgs<T> p,
             int* __restrict__ status) {
  constexpr bool SLOTS = TcTiles<WHICH>::SLOTS;
  constexpr bool A_K = WHICH == FFN_IN || WHICH == FFN_OUT, B_K = SLOTS;
  extern __shared__ char raw[];
  __shared__ __align__(8) uint64_t bars[3 * TC_STAGES + 6];
  __shared__ TcRanges of;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int failed;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t stages = (smem_at(raw) + 1023) & ~1023u;
  const uint32_t bar0 = smem_at(bars);
  auto land = [&](int s) { return bar0 + 8u * s; };                       // this block's copies of a stage with a ragged end
  auto ready = [&](int s) { return bar0 + 8u * (TC_STAGES + s); };        // first block: both blocks' stages are complete
  auto empty = [&](int s) { return bar0 + 8u * (2 * TC_STAGES + s); };    // the products have read a stage
  auto full = [&](int a) { return bar0 + 8u * (3 * TC_STAGES + a); };     // a tile's sums are complete
  auto taken = [&](int a) { return bar0 + 8u * (3 * TC_STAGES + 2 + a); };  // first block: both have read them
  const uint32_t done = bar0 + 8u * (3 * TC_STAGES + 4), never = done + 8u;

  if (threadIdx.x == 0) {
    failed = 0;
    for (int s = 0; s < TC_STAGES; ++s) {
      bar_init(land(s), 1);
      bar_init(ready(s), SLOTS ? 1 : 2);
      bar_init(empty(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      bar_init(full(a), 1);
      bar_init(taken(a), 2 * TC_EPILOGUE);
    }
    bar_init(done, 1);
    bar_init(never, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 3) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(&tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  TcTiles<WHICH> tiles;
  tiles.init(p.width, p.inner, SLOTS ? 1 : p.splits);
  if constexpr (WHICH != FFN_IN && WHICH != FFN_DH) {
    // everything before this point overlaps the product before, whose results are read from here on
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;");
  for (int e = threadIdx.x; e < p.experts; e += TC_THREADS) {
    const SlotRange r = slot_range(p.offsets, e, p.slots);
    of.lo[e] = (int)r.lo;
    of.hi[e] = (int)r.hi;
  }
  if (SLOTS) {
    __syncthreads();
    // An expert's tiles are of one size.  (Narrower ones for all experts, chosen by a cost of columns and rounds so that the
    // pairs' last round would be fuller, took between 2 % less and 4 % more time over ten shapes.)
    for (int e = threadIdx.x; e < p.experts; e += TC_THREADS) {
      const unsigned rows = of.hi[e] - of.lo[e], count = (rows + 255) / 256;  // rows + count: up to 2^31 + 2^23
      const unsigned wide = count > 1 ? ((rows + count - 1) / count + 31) & ~31u : 256;
      of.wide[e] = (short)wide;
      of.prefix[e + 1] = (int)((rows + wide - 1) / wide);
    }
  }
  if (SLOTS) {
    __syncthreads();
    if (warp == 0) {
      int before = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 32) {
        int x = e0 + lane < p.experts ? of.prefix[e0 + lane + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (e0 + lane < p.experts) of.prefix[e0 + lane + 1] = before + x;
        before += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) of.prefix[0] = 0;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && (WHICH == FFN_IN || WHICH == FFN_DH)) *status = ERC_OK;
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_arrive_wait();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base;
  const int total = SLOTS ? of.prefix[p.experts] * tiles.m_tiles : p.experts * tiles.splits * tiles.m_tiles * tiles.n_tiles;
  const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
  const int m_block = rank * TC_HALF;

  if (warp == 0) {
    if (lane == 0) {  // copies
      int s = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int at = first; ok && at < total; at += step) {
        const TcTile t = tiles.at(at, of, p.experts);
        const int m = t.m0 + m_block, n_half = t.n / 2;
        const uint32_t bytes = TC_OPERAND + (B_K ? TC_OPERAND : n_half * TC_K * 2);
        for (int b = 0; b < t.blocks; ++b) {
          if (!(ok = bar_wait(empty(s), phase ^ 1, &failed, p.patience))) break;
          const uint32_t dst = stages + s * TC_STAGE;
          const int k = b * TC_K;
          if constexpr (SLOTS) {
            const uint32_t bar = peer_address(ready(s), 0);
            if (rank == 0) bar_expect(ready(s), 2 * bytes);
            if constexpr (WHICH == FFN_IN) {
              copy_5d(dst, &map_a, bar, k, 0, 0, m / 16, t.expert);
            } else if constexpr (WHICH == FFN_OUT) {
              copy_3d(dst, &map_a, bar, k, m, t.expert);
            } else {
              copy_3d(dst, &map_a, bar, m, k, t.expert);
              copy_3d(dst + 8192, &map_a, bar, m + 64, k, t.expert);
            }
            copy_2d<true>(dst + TC_OPERAND, &map_b, bar, k, (int)(t.n0 + rank * n_half));
          } else {
            // all but a ragged end go to the first block's barrier; that one is passed on when its rows are in order
            const int n = (int)t.n0 + rank * n_half, row = (int)(t.k0 + k);
            auto boxes = [&](auto pair, uint32_t bar) {
              constexpr bool PAIR = decltype(pair)::value;
              copy_2d<PAIR>(dst, &map_a, bar, m, row);
              copy_2d<PAIR>(dst + 8192, &map_a, bar, m + 64, row);
              copy_2d<PAIR>(dst + TC_OPERAND, &map_b, bar, n, row);
              if (n_half > 64) copy_2d<PAIR>(dst + TC_OPERAND + 8192, &map_b, bar, n + 64, row);
            };
            if (t.k0 + k + TC_K > t.k1) {
              bar_expect(land(s), bytes);
              boxes(std::false_type(), land(s));
            } else {
              if (rank == 0) {
                bar_expect(ready(s), 2 * bytes);
                bar_arrive_cluster(peer_address(ready(s), 0));
              }
              boxes(std::true_type(), peer_address(ready(s), 0));
            }
          }
          if (++s == TC_STAGES) s = 0, phase ^= 1;
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {  // products
      int s = 0, a = 0;
      uint32_t phase = 0, a_phase = 0;
      bool ok = true;
      for (int at = first; ok && at < total; at += step) {
        const TcTile t = tiles.at(at, of, p.experts);
        if (t.blocks == 0) continue;
        const uint32_t idesc = (1u << 4) | (Half2<T>::FORMAT << 7) | (Half2<T>::FORMAT << 10) | ((A_K ? 0u : 1u) << 15) |
                               ((B_K ? 0u : 1u) << 16) | ((uint32_t)(t.n >> 3) << 17) | ((256u >> 4) << 24);
        if (!(ok = bar_wait(taken(a), a_phase ^ 1, &failed, p.patience))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + a * 256;
        for (int b = 0; b < t.blocks; ++b) {
          if (!(ok = bar_wait(ready(s), phase, &failed, p.patience))) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t da = operand_desc(stages + s * TC_STAGE, A_K), db = operand_desc(stages + s * TC_STAGE + TC_OPERAND, B_K);
#pragma unroll
          for (int k = 0; k < TC_K / 16; ++k)
            mma_pair(d, da + k * (A_K ? 32 >> 4 : 2048 >> 4), db + k * (B_K ? 32 >> 4 : 2048 >> 4), idesc, b > 0 || k > 0);
          commit_pair(empty(s));
          if (++s == TC_STAGES) s = 0, phase ^= 1;
        }
        if (!ok) break;
        commit_pair(full(a));
        if (++a == 2) a = 0, a_phase ^= 1;
      }
    }
  } else if (warp == 2) {
    // the ends of weight gradients: the rows of a box behind an expert's last slots belong to others, and become zeros
    if constexpr (!SLOTS) {
      int s = 0;
      uint32_t used = 0;  // bit s: the phase of land(s)
      for (int at = first; at < total; at += step) {
        const TcTile t = tiles.at(at, of, p.experts);
        if (t.blocks == 0) continue;
        s = (s + t.blocks - 1) % TC_STAGES;
        const int live = (int)(t.k1 - t.k0 - (int64_t)(t.blocks - 1) * TC_K);
        if (live < TC_K) {
          if (!__all_sync(0xffffffffu, bar_wait(land(s), used >> s & 1, &failed, p.patience))) break;
          used ^= 1u << s;
          const uint32_t base = stages + s * TC_STAGE;
          const int boxes = t.n > 128 ? 4 : 3;
          for (int x = 0; x < boxes; ++x)
            for (int i = live * 8 + lane; i < 512; i += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + x * 8192 + i * 16), "r"(0) : "memory");
          asm volatile("fence.proxy.async.shared::cta;\nfence.acq_rel.cluster;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(peer_address(ready(s), 0));
        }
        s = (s + 1) % TC_STAGES;
      }
    }
  } else if (warp == 3) {  // rows behind the last expert's, and what the first product left word of
    if constexpr (WHICH != FFN_IN && WHICH != FFN_DH) {
      if (blockIdx.x == 0) {
        int lost = 0;
        for (int i = lane; i < gridDim.x; i += 32) lost |= __ldcg(p.lost + i);
        if (lost) *status = ERC_ERR_TIMEOUT;
      }
    }
    if constexpr (WHICH == FFN_IN || WHICH == FFN_OUT || WHICH == FFN_DX) {
      T* out = WHICH == FFN_IN ? p.pre : WHICH == FFN_OUT ? p.y : p.dx;
      const int64_t row = (WHICH == FFN_IN ? 2 * (int64_t)p.inner : p.width) * sizeof(T) / 16;
      if (out)
        for (int64_t i = slots_used(p.offsets, p.experts, p.slots) * row + blockIdx.x * 32 + lane; i < p.slots * row;
             i += gridDim.x * 32)
          reinterpret_cast<uint4*>(out)[i] = make_uint4(0, 0, 0, 0);
    }
  } else {  // results
    constexpr int COLS = tc_cols(WHICH);
    const int quad = warp & 3, c0 = (warp - 4) / 4 * TC_PART;
    const bool keep = p.pre != nullptr;
    int a = 0;
    uint32_t a_phase = 0;
    bool ok = true;  // once a wait gave up this tile and the warp's later ones are NaN, and so is all that is made of them
    for (int at = first; at < total; at += step) {
      const TcTile t = tiles.at(at, of, p.experts);
      const int c1 = min(t.n, c0 + TC_PART);
      const TcOut out = tile_out<T, WHICH>(p, t, m_block, lane, quad);
      float v[COLS];
      PrePairs pre, next;  // DH: read a step before their use
      if (t.blocks == 0) {
#pragma unroll
        for (int i = 0; i < COLS; ++i) v[i] = 0.f;
#pragma unroll 1
        for (int c = c0; c < c1; c += COLS) write_columns<T, WHICH, ACT>(out, v, pre, c, lane, keep);
        continue;
      }
      auto read_ahead = [&](int c) {
        read_pre(out.pre_a, out.pre_b, out.at + (uint32_t)c / 2 * out.two, out.two, c, c < c1 ? out.live - out.col : 0, next);
      };
      if constexpr (WHICH == FFN_DH) read_ahead(c0);
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(full(a), a_phase, &failed, p.patience));
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t src = tmem + a * 256 + ((uint32_t)(quad * 32) << 16);
#pragma unroll 1
      for (int c = c0; c < c1; c += COLS) {
        if (ok) {
          read_tmem<COLS>(src + c, v);
        } else {
#pragma unroll
          for (int i = 0; i < COLS; ++i) v[i] = NAN;
        }
        if constexpr (WHICH == FFN_DH) {
          pre = next;
          read_ahead(c + COLS);
        }
        read_tmem_done();
        if (c + COLS >= c1) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (ok && lane == 0) bar_arrive_cluster(peer_address(taken(a), 0));
        }
        write_columns<T, WHICH, ACT>(out, v, pre, c, lane, keep);
      }
      if (c0 >= c1) {
        __syncwarp();
        if (ok && lane == 0) bar_arrive_cluster(peer_address(taken(a), 0));
      }
      if (++a == 2) a = 0, a_phase ^= 1;
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (failed) {
    if (threadIdx.x == 32 && rank == 0) {  // the thread that issued the products
      commit_pair(done);
      bar_poll(done, 0, TcPatience(), TC_WAIT, nullptr);
    }
    __syncthreads();
    // nothing arrives at this barrier, so this is a pause, for the copies
    if (threadIdx.x == 0) bar_poll(never, 0, TcPatience(0x7fffffffu), TC_COPIES, nullptr);
    __syncthreads();
  }
  cluster_arrive_wait();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 3) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  if (threadIdx.x == 0) {
    if (WHICH == FFN_IN || WHICH == FFN_DH)
      p.lost[blockIdx.x] = failed;
    else if (failed)
      *status = ERC_ERR_TIMEOUT;
  }
}

// ---- host side
// a tensor map of 16-bit elements; dims, strides (bytes, of all but the first) and box as given.  False when refused.
bool tc_encode(CUtensorMap* map, bool bf16, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
               const uint32_t* box);

template <class T, int WHICH>
erc_status ffn_tc_launch(const FfnArgs<T>& p, int* status, cudaStream_t s) {
  const uint64_t D = p.width, F = p.inner, E = p.experts, S = p.slots;
  constexpr bool BF = std::is_same<T, __nv_bfloat16>::value;
  CUtensorMap a, b;
  bool good = true;
  if constexpr (WHICH == FFN_IN) {
    // features in groups of 8, gates and factors of a group next to each other
    const uint64_t dims[5] = {D, 8, 2, F / 8, E}, strides[4] = {2 * D, 2 * D * F, 16 * D, 4 * D * F};
    const uint32_t box[5] = {TC_K, 8, 2, 8, 1};
    good = tc_encode(&a, BF, p.w_in, 5, dims, strides, box);
  } else if constexpr (WHICH == FFN_OUT || WHICH == FFN_DH) {
    const uint64_t dims[3] = {F, D, E}, strides[2] = {2 * F, 2 * D * F};
    const uint32_t box[3] = {TC_K, WHICH == FFN_OUT ? (uint32_t)TC_HALF : (uint32_t)TC_K, 1};
    good = tc_encode(&a, BF, p.w_out, 3, dims, strides, box);
  } else if constexpr (WHICH == FFN_DX) {
    const uint64_t dims[3] = {D, 2 * F, E}, strides[2] = {2 * D, 4 * D * F};
    const uint32_t box[3] = {TC_K, TC_K, 1};
    good = tc_encode(&a, BF, p.w_in, 3, dims, strides, box);
  } else {
    const uint64_t width = WHICH == FFN_DWIN ? D : F;
    const uint64_t dims[2] = {width, S}, strides[1] = {2 * width};
    const uint32_t box[2] = {TC_K, TC_K};
    good = tc_encode(&a, BF, WHICH == FFN_DWIN ? p.x : p.h, 2, dims, strides, box);
  }
  const uint64_t row = WHICH == FFN_IN || WHICH == FFN_DH || WHICH == FFN_DWOUT ? D : WHICH == FFN_OUT ? F : 2 * F;
  const void* from = WHICH == FFN_IN ? p.x : WHICH == FFN_OUT ? p.h : WHICH == FFN_DH || WHICH == FFN_DWOUT ? p.dy : p.dpre;
  const uint64_t dims[2] = {row, S}, strides[1] = {2 * row};
  const uint32_t box[2] = {TC_K, WHICH <= FFN_DX ? (uint32_t)TC_HALF : (uint32_t)TC_K};
  good = good && tc_encode(&b, BF, from, 2, dims, strides, box);
  if (!good) return set_error(ERC_ERR_CUDA, "a tensor map of the expert products was refused");
  // the activation is fixed at compile time: with all three in one kernel the unrolled columns do not fit the
  // instruction cache (DH of 80000 slots, 64 experts, 512 x 1024: 1048 us)
  constexpr bool ACTS = WHICH == FFN_IN || WHICH == FFN_DH;
  auto kernel = k_ffn_tc<T, WHICH, ERC_ACT_SILU>;
  if constexpr (ACTS) {
    if (p.act == ERC_ACT_GELU) kernel = k_ffn_tc<T, WHICH, ERC_ACT_GELU>;
    if (p.act == ERC_ACT_RELU) kernel = k_ffn_tc<T, WHICH, ERC_ACT_RELU>;
  }
  ERC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TC_SMEM));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tc_blocks());
  cfg.blockDim = dim3(TC_THREADS);
  cfg.dynamicSmemBytes = TC_SMEM;
  cfg.stream = s;
  cudaLaunchAttribute after[1];
  after[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  after[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = after;
  cfg.numAttrs = ACTS ? 0 : 1;  // the first product of a call starts when the work before the call is done
  ERC_CUDA(cudaLaunchKernelEx(&cfg, kernel, a, b, p, status));
  count_launches(1);
  return ERC_OK;
}

// the products of a type, in a translation unit of their own
#define ERC_FFN_TC_PRODUCTS(T)                                                                             \
  template <>                                                                                              \
  erc_status ffn_tc_product<T>(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s) {       \
    switch (which) {                                                                                       \
      case FFN_IN: return ffn_tc_launch<T, FFN_IN>(p, status, s);                                          \
      case FFN_OUT: return ffn_tc_launch<T, FFN_OUT>(p, status, s);                                        \
      case FFN_DH: return ffn_tc_launch<T, FFN_DH>(p, status, s);                                          \
      case FFN_DX: return ffn_tc_launch<T, FFN_DX>(p, status, s);                                          \
      case FFN_DWIN: return ffn_tc_launch<T, FFN_DWIN>(p, status, s);                                      \
      default: return ffn_tc_launch<T, FFN_DWOUT>(p, status, s);                                           \
    }                                                                                                      \
  }

}  // namespace erc
