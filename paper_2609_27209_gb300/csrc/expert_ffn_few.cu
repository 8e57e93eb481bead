// expert_ffn_few.cu -- the gated feed-forward block for a handful of slots (single tokens): the weights of the
// experts that have rows are read once, and that is what it costs.
//
// A warp takes four weight rows (IN: the gates and factors of two features; OUT: four results) and up to 8 slots at
// a time.  A lane multiplies its 16-byte pieces of the weights with the slots' pieces (from L1), so 32 lanes end
// with parts of up to 32 sums; halving steps leave sum i in lane i (31 shuffles for 32 sums).  OUT asks for its
// weights while IN still runs, and waits for h only then.
//
// 14 slots over 8 experts of 512 x 1024 bf16 (25 MB of weights, 3.7 us of copying): 13.5 us; one slot of one expert of
// 2048 x 2048 (25 MB) 11.5; in float32 19 and 18.7 (7.4).  A call takes 20 to 22, which is the binding's and the launches'
// time.  What bounds them is latency: offsets, weights, slots and the halving steps follow each other, with 128 and
// 64 blocks (2048 rows) for 152 SMs, issue active in 0.05 to 0.15 of the cycles, and, with few slots over many experts, blocks
// without any.
#include "expert_ffn.cuh"

namespace erc {
namespace {

constexpr int WT = 256;  // threads
constexpr int WW = WT / 32;
constexpr int WR = 4;    // weight rows of a warp

// v[0 .. COUNT): the warp's parts of COUNT sums (a power of two, at most 32).  Lane i ends with sum i mod COUNT.
template <int COUNT>
__device__ __forceinline__ float scatter_sums(float* v, int lane) {
#pragma unroll
  for (int n = COUNT; n > 1; n /= 2) {
    const bool upper = lane & (n / 2);
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float give = upper ? v[i] : v[i + n / 2], keep = upper ? v[i + n / 2] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, n / 2);
    }
  }
  float s = v[0];
#pragma unroll
  for (int o = 16; o >= COUNT; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

template <class T>
union FewPiece {
  uint4 raw;
  T t[16 / sizeof(T)];
  __device__ FewPiece() {}
};

// lane l gets sum (slot l / 4 mod R, weight row l mod 4) over `depth` elements; of slots from `rows` on the last one's
template <class T, int R>
__device__ __forceinline__ float few_sums(const T* const* w, const T* x, int rows, int depth, int lane) {
  constexpr int N = 16 / sizeof(T);
  float acc[R * WR];
#pragma unroll
  for (int i = 0; i < R * WR; ++i) acc[i] = 0.f;
#pragma unroll 2
  for (int k = lane * N; k < depth; k += 32 * N) {
    FewPiece<T> a[WR];
#pragma unroll
    for (int j = 0; j < WR; ++j) a[j].raw = __ldg(reinterpret_cast<const uint4*>(w[j] + k));
#pragma unroll
    for (int r = 0; r < R; ++r) {
      FewPiece<T> b;
      b.raw = *reinterpret_cast<const uint4*>(x + (int64_t)min(r, rows - 1) * depth + k);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float xv = to_f32(b.t[i]);
#pragma unroll
        for (int j = 0; j < WR; ++j) acc[r * WR + j] = fmaf(to_f32(a[j].t[i]), xv, acc[r * WR + j]);
      }
    }
  }
  return scatter_sums<R * WR>(acc, lane);
}

template <class T, int WHICH>
__global__ void __launch_bounds__(WT) k_ffn_few(const FfnArgs<T> p, int* __restrict__ status) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t D = p.width, F = p.inner;
  const int e = blockIdx.y;
  const int64_t thread = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * WT + threadIdx.x;
  const int64_t threads = (int64_t)gridDim.x * gridDim.y * WT;
  asm volatile("griddepcontrol.launch_dependents;");
  if (WHICH == FFN_IN && thread == 0) *status = ERC_OK;
  const int64_t used = slots_used(p.offsets, p.experts, p.slots);
  if (WHICH == FFN_IN && p.pre) zero_slots(p.pre, used, p.slots, 2 * F, thread, threads);
  if (WHICH == FFN_OUT) zero_slots(p.y, used, p.slots, D, thread, threads);
  const SlotRange s = slot_range(p.offsets, e, p.slots);
  const int depth = WHICH == FFN_IN ? p.width : p.inner;
  const int first = (blockIdx.x * WW + warp) * (WHICH == FFN_IN ? WR / 2 : WR);  // feature, or result
  const int rows = WHICH == FFN_IN ? p.inner : p.width;
  const bool some = s.lo < s.hi && first < rows;
  const T* w[WR];
#pragma unroll
  for (int j = 0; j < WR; ++j) {
    if (WHICH == FFN_IN)
      w[j] = p.w_in + (e * 2 * F + (j / 2) * F + min(first + j % 2, rows - 1)) * D;
    else
      w[j] = p.w_out + (e * D + min(first + j, rows - 1)) * F;
  }
  if constexpr (WHICH == FFN_OUT) {
    if (some)
      for (int k = lane * 64; k < depth; k += 32 * 64)  // a lane asks for 128 or 256 bytes of each row
#pragma unroll
        for (int j = 0; j < WR; ++j) {
          asm volatile("prefetch.global.L2 [%0];" ::"l"(w[j] + k));
          if (sizeof(T) == 4 && k + 32 < depth) asm volatile("prefetch.global.L2 [%0];" ::"l"(w[j] + k + 32));
        }
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }
  if (!some) return;
  const T* x = WHICH == FFN_IN ? p.x : p.h;
  for (int64_t r0 = s.lo; r0 < s.hi;) {
    const int R = (int)min(s.hi - r0, (int64_t)8);
    const T* from = x + r0 * depth;
    const float sum = R > 4    ? few_sums<T, 8>(w, from, R, depth, lane)
                      : R > 2  ? few_sums<T, 4>(w, from, R, depth, lane)
                      : R == 2 ? few_sums<T, 2>(w, from, R, depth, lane)
                               : few_sums<T, 1>(w, from, R, depth, lane);
    const int64_t row = r0 + lane / WR;
    const int j = lane % WR;
    if constexpr (WHICH == FFN_IN) {
      const float up = __shfl_xor_sync(0xffffffffu, sum, 2);  // lanes of gates: j 0 and 1
      const int f = first + j % 2;
      if (lane < R * WR && f < rows) {
        if (j < 2) p.h[row * F + f] = from_f32<T>(act_value(p.act, sum) * up);
        if (p.pre) p.pre[row * 2 * F + (j / 2) * F + f] = from_f32<T>(sum);
      }
    } else {
      if (lane < R * WR && first + j < rows) p.y[row * D + first + j] = from_f32<T>(sum);
    }
    r0 += R;
  }
}

template <class T, int WHICH>
erc_status few_launch(const FfnArgs<T>& p, int* status, cudaStream_t s) {
  const int each = WW * (WHICH == FFN_IN ? WR / 2 : WR), rows = WHICH == FFN_IN ? p.inner : p.width;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((rows + each - 1) / each, p.experts);
  cfg.blockDim = dim3(WT);
  cfg.stream = s;
  cudaLaunchAttribute after[1];
  after[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  after[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = after;
  cfg.numAttrs = WHICH == FFN_OUT ? 1 : 0;
  ERC_CUDA(cudaLaunchKernelEx(&cfg, k_ffn_few<T, WHICH>, p, status));
  count_launches(1);
  return ERC_OK;
}

}  // namespace

template <class T>
erc_status ffn_few_product(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s) {
  return which == FFN_IN ? few_launch<T, FFN_IN>(p, status, s) : few_launch<T, FFN_OUT>(p, status, s);
}
template erc_status ffn_few_product(FfnProduct, const FfnArgs<float>&, int*, cudaStream_t);
template erc_status ffn_few_product(FfnProduct, const FfnArgs<__nv_bfloat16>&, int*, cudaStream_t);
template erc_status ffn_few_product(FfnProduct, const FfnArgs<__half>&, int*, cudaStream_t);

}  // namespace erc
