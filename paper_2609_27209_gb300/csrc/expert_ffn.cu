// expert_ffn.cu -- the gated feed-forward block of experts: the C entry points, and its products on
// the float32 units, for every type and size (the tensor cores take the 16-bit types whose rows are
// whole 16-byte pieces, expert_ffn_tc.cuh).
//
// A product is C(i, j) = sum_k A(i, k) B(j, k) in tiles of 64 or 128 rows and columns by a depth of 16, twice
// buffered in shared memory.  A thread keeps 4 x 4 or 8 x 8 sums in registers, as groups of 4 rows and 4 columns 64
// apart.  In IN the second group of columns holds the factors of the first one's features.  Sums run over k in order,
// 256 at a time.
// Bound by issue (a product and its share of the shared-memory reads are instructions of their own) and by the tiles'
// rounds: 8192 slots of 1024 x 1024 float32, 43 to 44 TFLOP/s forward and 41 backward (library products: 45 to 57, by layout,
// and 50 to 57).
#include <initializer_list>

#include "expert_ffn.cuh"

namespace erc {
namespace {

constexpr int FT = 256;  // threads
constexpr int FM = 64;   // rows of a group: 16 threads by 4
constexpr int FK = 16;

// an operand: element (i, k) at p[i * row + k * step], i < rows.  One of row and step is 1.  With `twin` rows from FM of a
// tile on are those of the first FM, `twin` elements further (the factors of IN).
template <class T>
struct Operand {
  const T* p;
  int64_t row, step;
  int64_t rows;
  int64_t twin;
};

// E neighbouring elements of an operand's tile (GROUPS * FM rows by FK) for each thread; CONTIG: k is the contiguous index
template <int GROUPS, bool CONTIG>
struct Slice {
  static constexpr int E = GROUPS * FM * FK / FT;
  int i, k;
  __device__ __forceinline__ Slice() {
    if (CONTIG) {
      i = threadIdx.x / (FK / E);
      k = threadIdx.x % (FK / E) * E;
    } else {
      k = threadIdx.x / (GROUPS * FM / E);
      i = threadIdx.x % (GROUPS * FM / E) * E;
    }
  }
  template <class T>
  __device__ __forceinline__ void load(const Operand<T>& a, int64_t i0, int64_t k0, int64_t depth, float* r) const {
    int64_t row = i0 + i, shift = 0;
    if (a.twin && i >= FM) row -= FM, shift = a.twin;
    const int64_t at = k0 + k;
    const T* p = a.p + shift + row * a.row + at * a.step;
    constexpr int BYTES = E * sizeof(T) < 16 ? E * sizeof(T) : 16, PER = BYTES / sizeof(T);
    const bool whole = CONTIG ? row < a.rows && at + E <= depth : row + E <= a.rows && at < depth;
    if (whole && reinterpret_cast<uintptr_t>(p) % BYTES == 0) {
#pragma unroll
      for (int j = 0; j < E; j += PER) {
        union Piece {
          uint4 q;
          uint2 d;
          T t[16 / sizeof(T)];
          __device__ Piece() {}
        } v;
        if constexpr (BYTES == 16)
          v.q = __ldg(reinterpret_cast<const uint4*>(p + j));
        else
          v.d = __ldg(reinterpret_cast<const uint2*>(p + j));
#pragma unroll
        for (int q = 0; q < PER; ++q) r[j + q] = to_f32(v.t[q]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const bool in = CONTIG ? row < a.rows && at + j < depth : row + j < a.rows && at < depth;
        r[j] = in ? to_f32(p[j]) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void keep(float (*s)[GROUPS * FM + 4], const float* r) const {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      if (CONTIG)
        s[k + j][i] = r[j];
      else
        s[k][i + j] = r[j];
    }
  }
};

// Sums of FLUSH products go to a second set of sums.  Terms of mixed signs leave a sum of n of them off by some
// 2^-24 sqrt(n / 6) of its size; this way by 2^-24 sqrt((256 + n / 256) / 6), where the second part, of the second
// sums, is the larger one from 65536 terms on (2000 slots of 900 x 1000, three experts, the
// gradient of x: 9.7e-7 -> 4.1e-7 of its norm; 8192 x 1024 x 1024: forward 1186 -> 1170 us, gradient 2426 -> 2518 us).
// A weight gradient in parts has n slots of a part and the parts, up to 64, on top.
// It lies in shared memory: in registers it would leave room for fewer blocks (1000 slots of 500 x 300, gradient: 193
// instead of 155 us).
constexpr int FLUSH = 256;
template <int RG, int CG>
struct Tiles {
  float a[2][FK][RG * FM + 4];
  float b[2][FK][CG * FM + 4];
  float held[16 * RG * CG][FT];
};

// the thread's sums: rows i0 + 64 g + 4 (tid / 16) + ., columns j0 + 64 q + 4 (tid % 16) + .
template <class T, bool CA, bool CB, int RG, int CG>
__device__ __forceinline__ void product(Tiles<RG, CG>& s, const Operand<T>& a, const Operand<T>& b, int64_t i0, int64_t j0,
                                        int64_t depth, float (*acc)[4 * CG]) {
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  const Slice<RG, CA> sa;
  const Slice<CG, CB> sb;
#pragma unroll
  for (int i = 0; i < 4 * RG; ++i)
#pragma unroll
    for (int j = 0; j < 4 * CG; ++j) acc[i][j] = 0.f;
  const bool flushes = depth > FLUSH;
  if (flushes)
#pragma unroll
    for (int i = 0; i < 16 * RG * CG; ++i) s.held[i][threadIdx.x] = 0.f;
  float ra[Slice<RG, CA>::E], rb[Slice<CG, CB>::E];
  sa.load(a, i0, 0, depth, ra);
  sb.load(b, j0, 0, depth, rb);
  sa.keep(s.a[0], ra);
  sb.keep(s.b[0], rb);
  __syncthreads();
  int at = 0;
  for (int64_t k0 = 0; k0 < depth; k0 += FK) {
    const bool more = k0 + FK < depth;
    if (more) {
      sa.load(a, i0, k0 + FK, depth, ra);
      sb.load(b, j0, k0 + FK, depth, rb);
    }
#pragma unroll
    for (int k = 0; k < FK; ++k) {
      float xa[4 * RG], xb[4 * CG];
#pragma unroll
      for (int g = 0; g < RG; ++g)
        *reinterpret_cast<float4*>(xa + 4 * g) = *reinterpret_cast<const float4*>(&s.a[at][k][FM * g + 4 * ty]);
#pragma unroll
      for (int g = 0; g < CG; ++g)
        *reinterpret_cast<float4*>(xb + 4 * g) = *reinterpret_cast<const float4*>(&s.b[at][k][FM * g + 4 * tx]);
#pragma unroll
      for (int i = 0; i < 4 * RG; ++i)
#pragma unroll
        for (int j = 0; j < 4 * CG; ++j) acc[i][j] = fmaf(xa[i], xb[j], acc[i][j]);
    }
    if (more) {
      sa.keep(s.a[at ^ 1], ra);
      sb.keep(s.b[at ^ 1], rb);
    }
    __syncthreads();
    at ^= 1;
    if (flushes && (k0 / FK + 1) % (FLUSH / FK) == 0) {
#pragma unroll
      for (int i = 0; i < 4 * RG; ++i)
#pragma unroll
        for (int j = 0; j < 4 * CG; ++j) {
          s.held[i * 4 * CG + j][threadIdx.x] += acc[i][j];
          acc[i][j] = 0.f;
        }
    }
  }
  if (flushes)
#pragma unroll
    for (int i = 0; i < 4 * RG; ++i)
#pragma unroll
      for (int j = 0; j < 4 * CG; ++j) acc[i][j] += s.held[i * 4 * CG + j][threadIdx.x];
}

template <int RG, int CG>
__device__ __forceinline__ Tiles<RG, CG>& tiles_of() {
  extern __shared__ __align__(16) char tiles[];
  return *reinterpret_cast<Tiles<RG, CG>*>(tiles);
}

// the expert and rows of the t-th tile of `high` slots, experts one after another; false past the last
__device__ __forceinline__ bool find_tile(const int64_t* offsets, int experts, int64_t slots, int high, int64_t t, int& expert,
                                          SlotRange& rows) {
  __shared__ int64_t warp_sum[FT / 32];
  __shared__ int found;
  __shared__ int64_t before_found;
  constexpr int PER = ERC_ROUTE_MAX_EXPERTS / FT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t count[PER], sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = threadIdx.x * PER + j;
    count[j] = 0;
    if (e < experts) {
      const SlotRange r = slot_range(offsets, e, slots);
      count[j] = (r.hi - r.lo + high - 1) / high;
    }
    sum += count[j];
  }
  int64_t upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (threadIdx.x == 0) found = -1;
  if (lane == 31) warp_sum[warp] = upto;
  __syncthreads();
  int64_t before = upto - sum;
  for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (t >= before && t < before + count[j]) {
      found = threadIdx.x * PER + j;
      before_found = before;
    }
    before += count[j];
  }
  __syncthreads();
  if (found < 0) return false;
  expert = found;
  rows = slot_range(offsets, expert, slots);
  rows.lo += (t - before_found) * high;
  return true;
}

// rows of a tile of slots against columns of a weight matrix
template <class T, int WHICH, int RG, int CG>
__global__ void __launch_bounds__(FT) k_ffn_slots(const FfnArgs<T> p) {
  Tiles<RG, CG>& s = tiles_of<RG, CG>();
  const int64_t D = p.width, F = p.inner;
  if (WHICH != FFN_DH) {
    const int64_t used = slots_used(p.offsets, p.experts, p.slots);
    const int64_t thread = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * FT + threadIdx.x;
    const int64_t threads = (int64_t)gridDim.x * gridDim.y * FT;
    if (WHICH == FFN_IN && p.pre) zero_slots(p.pre, used, p.slots, 2 * F, thread, threads);
    if (WHICH == FFN_OUT) zero_slots(p.y, used, p.slots, D, thread, threads);
    if (WHICH == FFN_DX) zero_slots(p.dx, used, p.slots, D, thread, threads);
  }
  int e;
  SlotRange r;
  if (!find_tile(p.offsets, p.experts, p.slots, RG * FM, blockIdx.x, e, r)) return;
  const int64_t j0 = (int64_t)blockIdx.y * (WHICH == FFN_IN ? FM : CG * FM);
  float acc[4 * RG][4 * CG];
  if constexpr (WHICH == FFN_IN) {
    const Operand<T> a = {p.x, D, 1, r.hi, 0}, b = {p.w_in + e * 2 * F * D, D, 1, F, F * D};
    product<T, true, true, RG, CG>(s, a, b, r.lo, j0, D, acc);
  } else if constexpr (WHICH == FFN_OUT) {
    const Operand<T> a = {p.h, F, 1, r.hi, 0}, b = {p.w_out + e * D * F, F, 1, D, 0};
    product<T, true, true, RG, CG>(s, a, b, r.lo, j0, F, acc);
  } else if constexpr (WHICH == FFN_DH) {
    const Operand<T> a = {p.dy, D, 1, r.hi, 0}, b = {p.w_out + e * D * F, 1, F, F, 0};
    product<T, true, false, RG, CG>(s, a, b, r.lo, j0, D, acc);
  } else {
    const Operand<T> a = {p.dpre, 2 * F, 1, r.hi, 0}, b = {p.w_in + e * 2 * F * D, 1, D, D, 0};
    product<T, true, false, RG, CG>(s, a, b, r.lo, j0, 2 * F, acc);
  }
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
#pragma unroll
  for (int i = 0; i < 4 * RG; ++i) {
    const int64_t row = r.lo + FM * (i / 4) + 4 * ty + i % 4;
    if (row >= r.hi) continue;
#pragma unroll
    for (int j = 0; j < (WHICH == FFN_IN ? 4 : 4 * CG); ++j) {
      const int64_t col = j0 + FM * (j / 4) + 4 * tx + j % 4;
      const float v = acc[i][j];
      if constexpr (WHICH == FFN_IN) {
        if (col >= F) continue;
        const float u = acc[i][4 + j];
        p.h[row * F + col] = from_f32<T>(act_value(p.act, v) * u);
        if (p.pre) {
          p.pre[row * 2 * F + col] = from_f32<T>(v);
          p.pre[row * 2 * F + F + col] = from_f32<T>(u);
        }
      } else if constexpr (WHICH == FFN_DH) {
        if (col >= F) continue;
        const float g = to_f32(p.pre_in[row * 2 * F + col]), u = to_f32(p.pre_in[row * 2 * F + F + col]);
        float value, slope;
        act_both(p.act, g, value, slope);
        p.dpre[row * 2 * F + col] = from_f32<T>(v * u * slope);
        p.dpre[row * 2 * F + F + col] = from_f32<T>(v * value);
        p.h[row * F + col] = from_f32<T>(value * u);
      } else {
        if (col < D) (WHICH == FFN_OUT ? p.y : p.dx)[row * D + col] = from_f32<T>(v);
      }
    }
  }
}

// a tile of an expert's weight gradient: the sum over its slots
template <class T, int WHICH, int RG, int CG>
__global__ void __launch_bounds__(FT) k_ffn_weights(const FfnArgs<T> p) {
  Tiles<RG, CG>& s = tiles_of<RG, CG>();
  const int64_t D = p.width, F = p.inner;
  const int e = blockIdx.z / p.splits, part = blockIdx.z - e * p.splits;
  const SlotRange r = split_range(slot_range(p.offsets, e, p.slots), part, p.splits);
  const int64_t i0 = (int64_t)blockIdx.y * (RG * FM), j0 = (int64_t)blockIdx.x * (CG * FM);
  const int64_t rows = WHICH == FFN_DWIN ? 2 * F : D, cols = WHICH == FFN_DWIN ? D : F;
  const Operand<T> a = {(WHICH == FFN_DWIN ? p.dpre : p.dy) + r.lo * rows, 1, rows, rows, 0};
  const Operand<T> b = {(WHICH == FFN_DWIN ? p.x : p.h) + r.lo * cols, 1, cols, cols, 0};
  float acc[4 * RG][4 * CG];
  product<T, false, false, RG, CG>(s, a, b, i0, j0, r.hi - r.lo, acc);
  T* out = (WHICH == FFN_DWIN ? p.dw_in : p.dw_out) + e * rows * cols;
  float* sums = p.splits > 1 ? p.partial + ((int64_t)part * p.experts + e) * rows * cols : nullptr;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
#pragma unroll
  for (int i = 0; i < 4 * RG; ++i)
#pragma unroll
    for (int j = 0; j < 4 * CG; ++j) {
      const int64_t row = i0 + FM * (i / 4) + 4 * ty + i % 4, col = j0 + FM * (j / 4) + 4 * tx + j % 4;
      if (row < rows && col < cols) {
        if (sums)
          sums[row * cols + col] = acc[i][j];
        else
          out[row * cols + col] = from_f32<T>(acc[i][j]);
      }
    }
}

// Whether a weight gradient of rows x cols takes tiles of 128: enough of them for every SM, or slots enough to split their
// sums until there are.  The whole float32 gradient with tiles of 64 / 128 (us).  It takes 128: one expert of 1024 x 1024,
// 8192 slots 2939 / 2511, 1024 slots 435 / 400; 8192 of 512 x 512, 780 / 663; 20000 of 200 x 200, 491 / 450; 20000 of 8 experts,
// 256 x 512, 1046 / 929.  It takes 64: 8192 of 96 x 96, 90 / 160; 30000 of 128 x 128, 240 / 264; 1000 of 500 x 300, 165 / 294;
// 4096 of 8 experts, 256 x 512, 234 / 239; 515 of 5 experts, 100 x 67, 43 / 60.
bool large_weights(int64_t slots, int experts, int64_t rows, int64_t cols) {
  const int64_t tiles = ((rows + 2 * FM - 1) / (2 * FM)) * ((cols + 2 * FM - 1) / (2 * FM)) * experts;
  if (tiles >= sm_count()) return true;
  return rows >= 96 && cols >= 96 && slots >= (int64_t)experts * 1024 && tiles * (slots / ((int64_t)experts * 512)) >= sm_count();
}

template <int RG, int CG, class K, class P>
erc_status launch_tiles(K kernel, dim3 grid, const P& p, cudaStream_t s) {
  constexpr size_t bytes = sizeof(Tiles<RG, CG>);
  // small calls are bound by the host, and what every launch may have needs no asking
  if constexpr (bytes > 48 * 1024)
    ERC_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  kernel<<<grid, FT, bytes, s>>>(p);
  return ERC_OK;
}

// tiles of 128 rows and columns where there is one for every SM, else of 64: a thread's 64 sums take half the
// shared-memory reads a product that 16 take, but few large tiles leave SMs idle
template <class T, int WHICH>
erc_status simple_launch(const FfnArgs<T>& p, cudaStream_t s) {
  const int64_t least = p.experts < p.slots ? p.experts : p.slots, busy = (int64_t)sm_count();
  if constexpr (WHICH <= FFN_DX) {
    const int64_t cols = WHICH == FFN_IN || WHICH == FFN_DH ? p.inner : p.width;
    const int64_t wide = WHICH == FFN_IN ? FM : 2 * FM;  // columns of a large tile
    const int64_t large = (p.slots / (2 * FM) + 1) * ((cols + wide - 1) / wide);
    if (large >= busy) {
      const int64_t tiles = p.slots / (2 * FM) + least;
      ERC_TRY((launch_tiles<2, 2>(k_ffn_slots<T, WHICH, 2, 2>, dim3((unsigned)tiles, (unsigned)((cols + wide - 1) / wide)), p, s)));
    } else {
      const int64_t tiles = p.slots / FM + least;
      constexpr int CG = WHICH == FFN_IN ? 2 : 1;
      ERC_TRY((launch_tiles<1, CG>(k_ffn_slots<T, WHICH, 1, CG>, dim3((unsigned)tiles, (unsigned)((cols + FM - 1) / FM)), p, s)));
    }
  } else {
    const int64_t rows = WHICH == FFN_DWIN ? 2 * (int64_t)p.inner : p.width, cols = WHICH == FFN_DWIN ? p.width : p.inner;
    const int64_t r2 = (rows + 2 * FM - 1) / (2 * FM), c2 = (cols + 2 * FM - 1) / (2 * FM);
    const unsigned deep = (unsigned)p.experts * p.splits;
    if (large_weights(p.slots, p.experts, rows, cols))
      ERC_TRY((launch_tiles<2, 2>(k_ffn_weights<T, WHICH, 2, 2>, dim3((unsigned)c2, (unsigned)r2, deep), p, s)));
    else
      ERC_TRY((launch_tiles<1, 1>(k_ffn_weights<T, WHICH, 1, 1>,
                                  dim3((unsigned)((cols + FM - 1) / FM), (unsigned)((rows + FM - 1) / FM), deep), p, s)));
  }
  count_launches(1);
  ERC_CUDA(cudaGetLastError());
  return ERC_OK;
}
template <class T>
erc_status simple_product(FfnProduct which, const FfnArgs<T>& p, cudaStream_t s) {
  switch (which) {
    case FFN_IN: return simple_launch<T, FFN_IN>(p, s);
    case FFN_OUT: return simple_launch<T, FFN_OUT>(p, s);
    case FFN_DH: return simple_launch<T, FFN_DH>(p, s);
    case FFN_DX: return simple_launch<T, FFN_DX>(p, s);
    case FFN_DWIN: return simple_launch<T, FFN_DWIN>(p, s);
    default: return simple_launch<T, FFN_DWOUT>(p, s);
  }
}

// ---- how a call's products run
enum FfnWay { FFN_SIMPLE, FFN_FEW, FFN_TENSOR };

// Few slots read the weights without the tensor cores.  IN + OUT, this way / by tiles (us, weights in L2):
//   one expert of 2048 x 2048       bfloat16: 4 slots 12 / 28, 8: 19 / 28, 16: 34 / 28; float32: 8: 23 / 230, 16: 44 / 231
//   8 experts of 512 x 1024         bfloat16: 16 slots 11 / 20, 32: 13 / 21, 64: 18 / 20; float32: 32: 15 / 87, 64: 22 / 87
//   64 experts of 1024 x 512        bfloat16: 32 slots 40 / 36, 64: 69 / 53; float32: 32: 51 / 207, 64: 87 / 379
// The bound is bfloat16's; float32, whose tiles are of 64 rows whatever is in them, would gain from a later one.
bool few_slots(const erc_ffn_shape* f) { return f->slots <= 8 || (f->slots <= 32 && f->slots <= 4 * f->experts); }
bool whole_pieces(const erc_ffn_shape* f) {
  const int piece = 16 / type_bytes(f->type);
  return f->width % piece == 0 && f->inner % piece == 0;
}
// Rows that are not whole pieces are copied into rows that are, for the tensor cores' sake: the copies cost some 20 us and
// three times the weights' bytes.  bfloat16, on the float32 units / this way (us, forward; gradient): 8192 slots of 1021 x
// 1023, 1440 / 86; 3750 / 189.  At the bounds: 100 slots of 1001 x 1001, 220 / 37; 334 / 66; 400 of 501 x 501, 117 / 31; 237 / 60;
// 400 slots of 8 experts, 511 x 511, 118 / 31; 206 / 59.  Below them it would pay too, at the price of the copies'
// workspace: 1000 slots of 201 x 201, 53 / 23; 256 / 52; 250 slots of 8 experts, 511 x 511, 109 / 29; 184 / 58.
bool worth_padding(const erc_ffn_shape* f) {
  return f->type != ERC_F32 && !whole_pieces(f) && f->slots >= 32 * (int64_t)f->experts &&
         (double)f->slots * f->width * f->inner >= 1e8;
}
// `all`: the bits of every pointer
FfnWay ffn_way(const erc_ffn_shape* f, uintptr_t all, bool forward) {
  if (worth_padding(f)) return FFN_TENSOR;
  if (all % 16 != 0 || !whole_pieces(f)) return FFN_SIMPLE;
  if (forward && few_slots(f)) return FFN_FEW;
  return f->type == ERC_F32 ? FFN_SIMPLE : FFN_TENSOR;
}

// Parts of an expert's slots in a weight gradient of rows x cols: few tiles would leave most SMs idle over a long sum
// (100000 slots of 32 x 64 bfloat16, the whole gradient: 986 us in one part, 111 to 126 in 64).
int weight_splits(const erc_ffn_shape* f, int64_t rows, int64_t cols, bool tensor) {
  const int64_t side = tensor ? 256 : large_weights(f->slots, f->experts, rows, cols) ? 2 * FM : FM;
  const int64_t most = tensor ? sm_count() / 2 : 2 * sm_count();
  const int64_t tiles = f->experts * ((rows + side - 1) / side) * ((cols + side - 1) / side);
  int64_t n = most / (tiles > 0 ? tiles : 1);
  const int64_t deep = f->slots / ((int64_t)f->experts * 512);
  if (n > deep) n = deep;
  return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

// the splits' sums, added in order and rounded once
template <class T>
__global__ void __launch_bounds__(FT) k_ffn_sum(const float* __restrict__ partial, int splits, int64_t count, T* __restrict__ out) {
  for (int64_t i = (int64_t)blockIdx.x * FT + threadIdx.x; i < count; i += (int64_t)gridDim.x * FT) {
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < splits; ++k) s += __ldcg(partial + k * count + i);
    out[i] = from_f32<T>(s);
  }
}

// dst [groups][rows_to][cols_to] from src [groups][rows_from][cols_from], zeros where src has none; several at once
template <class T>
struct Recast {
  const T* src;
  T* dst;
  int64_t groups;
  int rows_from, cols_from, rows_to, cols_to;
};
template <class T>
struct Recasts {
  Recast<T> job[5];
  int jobs = 0;
  void add(const T* src, T* dst, int64_t groups, int rows_from, int cols_from, int rows_to, int cols_to) {
    if (src && dst) job[jobs++] = {src, dst, groups, rows_from, cols_from, rows_to, cols_to};
  }
};
template <class T>
__global__ void __launch_bounds__(FT) k_ffn_recast(const Recasts<T> all) {
  const Recast<T> j = all.job[blockIdx.y];
  const int64_t rows = j.groups * j.rows_to;
  const int lane = threadIdx.x & 31;
  for (int64_t r = ((int64_t)blockIdx.x * FT + threadIdx.x) >> 5; r < rows; r += (int64_t)gridDim.x * (FT / 32)) {
    const int64_t g = r / j.rows_to;
    const int i = (int)(r - g * j.rows_to);
    const T* from = j.src + (g * j.rows_from + i) * j.cols_from;
    const int some = i < j.rows_from ? j.cols_from : 0;
#pragma unroll 4
    for (int c = lane; c < j.cols_to; c += 32) j.dst[r * j.cols_to + c] = c < some ? from[c] : from_f32<T>(0.f);
  }
}
template <class T>
erc_status recast(const Recasts<T>& all, cudaStream_t s) {
  if (all.jobs == 0) return ERC_OK;
  k_ffn_recast<T><<<dim3(sm_count() * 8, all.jobs), FT, 0, s>>>(all);
  count_launches(1);
  ERC_CUDA(cudaGetLastError());
  return ERC_OK;
}

template <class T>
erc_status ffn_product(FfnWay way, FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s) {
  if (way == FFN_FEW) return ffn_few_product<T>(which, p, status, s);
  if (way == FFN_TENSOR) {
    if constexpr (sizeof(T) == 2) ERC_TRY(ffn_tc_product<T>(which, p, status, s));
  } else {
    if (which == FFN_IN || which == FFN_DH) ERC_CUDA(cudaMemsetAsync(status, 0, sizeof(int), s));
    ERC_TRY(simple_product(which, p, s));
  }
  if (which >= FFN_DWIN && p.splits > 1) {
    const int64_t count = (int64_t)p.experts * p.width * p.inner * (which == FFN_DWIN ? 2 : 1);
    const int64_t blocks = (count + FT - 1) / FT, most = (int64_t)sm_count() * 8;
    k_ffn_sum<T><<<(unsigned)(blocks < most ? blocks : most), FT, 0, s>>>(p.partial, p.splits, count,
                                                                         which == FFN_DWIN ? p.dw_in : p.dw_out);
    count_launches(1);
    ERC_CUDA(cudaGetLastError());
  }
  return ERC_OK;
}

// what a call keeps in its workspace
template <class T>
struct FfnSpace {
  int *status, *lost;
  T *h, *dpre;
  float* partial;
  T *x, *dy, *pre, *w_in, *w_out, *y, *dx, *dw_in, *dw_out;  // rows of whole pieces
};
template <class T>
void plan_space(Arena& a, FfnSpace<T>& w, const erc_ffn_shape* f, bool backward) {
  const bool pad = worth_padding(f);
  const size_t S = f->slots, E = f->experts, D = pad ? (f->width + 7) / 8 * 8 : f->width, F = pad ? (f->inner + 7) / 8 * 8 : f->inner;
  w = {};
  w.status = a.take<int>(1);
  w.lost = a.take<int>(tc_blocks());
  w.h = a.take<T>(S * F);
  if (backward) {
    w.dpre = a.take<T>(S * 2 * F);
    size_t sums = 0;
    for (int tensor = 0; tensor < 2; ++tensor) {
      const size_t in = weight_splits(f, 2 * F, D, tensor), out = weight_splits(f, D, F, tensor);
      if (in > 1 && sums < in * E * 2 * F * D) sums = in * E * 2 * F * D;
      if (out > 1 && sums < out * E * F * D) sums = out * E * F * D;
    }
    w.partial = a.take<float>(sums);
  }
  if (!pad) return;
  w.x = a.take<T>(S * D);
  w.pre = a.take<T>(S * 2 * F);
  w.w_in = a.take<T>(E * 2 * F * D);
  w.w_out = a.take<T>(E * D * F);
  w.y = a.take<T>(S * D);
  if (!backward) return;
  w.dy = w.y;
  w.dx = a.take<T>(S * D);
  w.dw_in = a.take<T>(E * 2 * F * D);
  w.dw_out = a.take<T>(E * D * F);
}
size_t space_bytes(const erc_ffn_shape* f, bool backward) {
  Arena a(nullptr);
  if (f->type == ERC_F32) {
    FfnSpace<float> w;
    plan_space(a, w, f, backward);
  } else {
    FfnSpace<__half> w;
    plan_space(a, w, f, backward);
  }
  return a.used + 256;
}

erc_status check_shape(const erc_ffn_shape* f) {
  ERC_REQUIRE(f, "shape is required");
  ERC_REQUIRE(f->type >= ERC_F32 && f->type <= ERC_F16, "bad type %d", f->type);
  ERC_REQUIRE(f->act >= ERC_ACT_SILU && f->act <= ERC_ACT_RELU, "bad act %d", f->act);
  ERC_REQUIRE(f->slots >= 0 && f->slots <= 0x7fffffffLL, "slots must be in [0, 2^31)");
  ERC_REQUIRE(f->experts >= 1 && f->experts <= ERC_ROUTE_MAX_EXPERTS, "experts must be in [1, %d]", ERC_ROUTE_MAX_EXPERTS);
  ERC_REQUIRE(f->width >= 1 && f->width <= ERC_FFN_MAX_WIDTH && f->inner >= 1 && f->inner <= ERC_FFN_MAX_WIDTH,
              "width and inner must be in [1, %d]", ERC_FFN_MAX_WIDTH);
  return ERC_OK;
}
bool good_shape(const erc_ffn_shape* f) {
  return f && f->type >= ERC_F32 && f->type <= ERC_F16 && f->slots >= 0 && f->slots <= 0x7fffffffLL && f->experts >= 1 &&
         f->experts <= ERC_ROUTE_MAX_EXPERTS && f->width >= 1 && f->width <= ERC_FFN_MAX_WIDTH && f->inner >= 1 &&
         f->inner <= ERC_FFN_MAX_WIDTH;
}
uintptr_t any_bits(std::initializer_list<const void*> all) {
  uintptr_t v = 0;
  for (const void* p : all) v |= reinterpret_cast<uintptr_t>(p);
  return v;
}
void* align_ws(void* ws) {
  return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~uintptr_t(255));
}

}  // namespace
}  // namespace erc

using namespace erc;

extern "C" size_t erc_expert_ffn_workspace_size(const erc_ffn_shape* f) { return good_shape(f) ? space_bytes(f, false) : 0; }

extern "C" erc_status erc_expert_ffn(const erc_ffn_shape* f, const void* xs, const int64_t* offsets, const void* w_in,
                                     const void* w_out, void* y, void* pre, void* ws, size_t ws_bytes,
                                     erc_stream stream) {
  clear_error();
  ERC_TRY(check_shape(f));
  if (f->slots == 0) return ERC_OK;
  ERC_REQUIRE(xs && offsets && w_in && w_out && y, "null pointer");
  const uintptr_t all = any_bits({xs, w_in, w_out, y, pre});
  ERC_REQUIRE(all % type_bytes(f->type) == 0 && reinterpret_cast<uintptr_t>(offsets) % 8 == 0, "misaligned array");
  if (!ws || ws_bytes < space_bytes(f, false)) return set_error(ERC_ERR_CAPACITY, "workspace too small");
  const FfnWay way = ffn_way(f, all, true);
  const cudaStream_t s = as_stream(stream);
  return with_type(f->type, [&](auto t) {
    using T = decltype(t);
    Arena ar(align_ws(ws));
    FfnSpace<T> w;
    plan_space(ar, w, f, false);
    FfnArgs<T> p = {f->slots, f->experts, f->width, f->inner, f->act, offsets};
    p.x = static_cast<const T*>(xs);
    p.w_in = static_cast<const T*>(w_in);
    p.w_out = static_cast<const T*>(w_out);
    p.h = w.h;
    p.pre = static_cast<T*>(pre);
    p.y = static_cast<T*>(y);
    p.splits = 1;
    p.patience = TcPatience(wait_limit(0));
    p.lost = w.lost;
    const int D = p.width, F = p.inner, E = p.experts;
    if (w.x) {
      p.width = (D + 7) / 8 * 8;
      p.inner = (F + 7) / 8 * 8;
      Recasts<T> to;
      to.add(p.x, w.x, 1, (int)p.slots, D, (int)p.slots, p.width);
      to.add(p.w_in, w.w_in, 2 * E, F, D, p.inner, p.width);
      to.add(p.w_out, w.w_out, E, D, F, p.width, p.inner);
      ERC_TRY(recast(to, s));
      p.x = w.x;
      p.w_in = w.w_in;
      p.w_out = w.w_out;
      p.pre = pre ? w.pre : nullptr;
      p.y = w.y;
    }
    ERC_TRY(ffn_product(way, FFN_IN, p, w.status, s));
    ERC_TRY(ffn_product(way, FFN_OUT, p, w.status, s));
    if (!w.x) return ERC_OK;
    Recasts<T> back;
    back.add(w.y, static_cast<T*>(y), 1, (int)p.slots, p.width, (int)p.slots, D);
    back.add(w.pre, static_cast<T*>(pre), 2 * p.slots, 1, p.inner, 1, F);
    return recast(back, s);
  });
}

extern "C" size_t erc_expert_ffn_backward_workspace_size(const erc_ffn_shape* f) {
  return good_shape(f) ? space_bytes(f, true) : 0;
}

extern "C" erc_status erc_expert_ffn_backward(const erc_ffn_shape* f, const void* dy, const void* xs, const void* pre,
                                              const int64_t* offsets, const void* w_in, const void* w_out, void* dxs,
                                              void* dw_in, void* dw_out, void* ws, size_t ws_bytes, erc_stream stream) {
  clear_error();
  ERC_TRY(check_shape(f));
  if (!dxs && !dw_in && !dw_out) return ERC_OK;
  const cudaStream_t s = as_stream(stream);
  if (f->slots == 0) {
    const size_t bytes = (size_t)f->experts * f->width * f->inner * type_bytes(f->type);
    if (dw_in) ERC_CUDA(cudaMemsetAsync(dw_in, 0, 2 * bytes, s));
    if (dw_out) ERC_CUDA(cudaMemsetAsync(dw_out, 0, bytes, s));
    return ERC_OK;
  }
  ERC_REQUIRE(dy && pre && offsets && w_out && (xs || !dw_in) && (w_in || !dxs), "null pointer");
  const uintptr_t all = any_bits({dy, xs, pre, w_in, w_out, dxs, dw_in, dw_out});
  ERC_REQUIRE(all % type_bytes(f->type) == 0 && reinterpret_cast<uintptr_t>(offsets) % 8 == 0, "misaligned array");
  if (!ws || ws_bytes < space_bytes(f, true)) return set_error(ERC_ERR_CAPACITY, "workspace too small");
  const FfnWay way = ffn_way(f, all, false);
  return with_type(f->type, [&](auto t) {
    using T = decltype(t);
    Arena ar(align_ws(ws));
    FfnSpace<T> w;
    plan_space(ar, w, f, true);
    FfnArgs<T> p = {f->slots, f->experts, f->width, f->inner, f->act, offsets};
    p.x = static_cast<const T*>(xs);
    p.w_in = static_cast<const T*>(w_in);
    p.w_out = static_cast<const T*>(w_out);
    p.dy = static_cast<const T*>(dy);
    p.pre_in = static_cast<const T*>(pre);
    p.dpre = w.dpre;
    p.h = w.h;
    p.dx = static_cast<T*>(dxs);
    p.dw_in = static_cast<T*>(dw_in);
    p.dw_out = static_cast<T*>(dw_out);
    p.partial = w.partial;
    p.splits = 1;
    p.patience = TcPatience(wait_limit(0));
    p.lost = w.lost;
    const int D = p.width, F = p.inner, E = p.experts;
    if (w.x) {
      p.width = (D + 7) / 8 * 8;
      p.inner = (F + 7) / 8 * 8;
      Recasts<T> to;
      to.add(p.dy, w.dy, 1, (int)p.slots, D, (int)p.slots, p.width);
      to.add(p.pre_in, w.pre, 2 * p.slots, 1, F, 1, p.inner);
      to.add(p.w_out, w.w_out, E, D, F, p.width, p.inner);
      if (dw_in) to.add(p.x, w.x, 1, (int)p.slots, D, (int)p.slots, p.width);
      if (dxs) to.add(p.w_in, w.w_in, 2 * E, F, D, p.inner, p.width);
      ERC_TRY(recast(to, s));
      p.dy = w.dy;
      p.pre_in = w.pre;
      p.x = w.x;
      p.w_in = w.w_in;
      p.w_out = w.w_out;
      p.dx = dxs ? w.dx : nullptr;
      p.dw_in = dw_in ? w.dw_in : nullptr;
      p.dw_out = dw_out ? w.dw_out : nullptr;
    }
    ERC_TRY(ffn_product(way, FFN_DH, p, w.status, s));
    if (p.dx) ERC_TRY(ffn_product(way, FFN_DX, p, w.status, s));
    p.splits = weight_splits(f, 2 * p.inner, p.width, way == FFN_TENSOR);
    if (p.dw_in) ERC_TRY(ffn_product(way, FFN_DWIN, p, w.status, s));
    p.splits = weight_splits(f, p.width, p.inner, way == FFN_TENSOR);
    if (p.dw_out) ERC_TRY(ffn_product(way, FFN_DWOUT, p, w.status, s));
    if (!w.x) return ERC_OK;
    Recasts<T> back;
    back.add(w.dx, static_cast<T*>(dxs), 1, (int)p.slots, p.width, (int)p.slots, D);
    back.add(w.dw_in, static_cast<T*>(dw_in), 2 * E, p.inner, p.width, F, D);
    back.add(w.dw_out, static_cast<T*>(dw_out), E, p.width, p.inner, D, F);
    return recast(back, s);
  });
}
