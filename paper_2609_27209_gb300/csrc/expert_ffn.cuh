// expert_ffn.cuh -- what the gated feed-forward block's two paths share: the float32 units' (all types
// and sizes, expert_ffn.cu) and the tensor cores' (expert_ffn_tc.cu).
//
// With h = act(a) b and s a slot of expert e, the block is six products:
//   IN    (a, b)[s] = w_in[e] x[s]           OUT   y[s] = w_out[e] h[s]
//   DH    dh[s] = dy[s] w_out[e], then da = dh b act'(a), db = dh act(a), and h again from (a, b)
//   DX    dx[s] = (da, db)[s] w_in[e]
//   DWIN  dw_in[e] = sum_s (da, db)[s] x[s]^T     DWOUT  dw_out[e] = sum_s dy[s] h[s]^T
#pragma once

#include "choice.cuh"

namespace erc {

enum FfnProduct { FFN_IN, FFN_OUT, FFN_DH, FFN_DX, FFN_DWIN, FFN_DWOUT };

// the arrays of all six; a product uses those that it names
template <class T>
struct FfnArgs {
  int64_t slots;
  int experts, width, inner, act;
  const int64_t* offsets;
  const T* x;
  const T* w_in;
  const T* w_out;
  const T* dy;
  const T* pre_in;  // (a, b), read
  T* pre;           // (a, b), written; may be null
  T* h;             // act(a) b
  T* dpre;          // (da, db)
  T* y;
  T* dx;
  T* dw_in;
  T* dw_out;
};

// [lo, hi) of an expert; whatever the offsets hold, it lies in [0, slots]
struct SlotRange {
  int64_t lo, hi;
};
__device__ __forceinline__ SlotRange slot_range(const int64_t* offsets, int e, int64_t slots) {
  int64_t lo = __ldg(offsets + e), hi = __ldg(offsets + e + 1);
  lo = lo < 0 ? 0 : lo > slots ? slots : lo;
  hi = hi < lo ? lo : hi > slots ? slots : hi;
  return {lo, hi};
}
__device__ __forceinline__ int64_t slots_used(const int64_t* offsets, int experts, int64_t slots) {
  const int64_t v = __ldg(offsets + experts);
  return v < 0 ? 0 : v > slots ? slots : v;
}


// act(a), and act'(a).  The normal distribution function comes from erfc, which keeps its relative accuracy in the lower
// tail; the sigmoid from the hardware's 2^x and 1 / x (a few units in the last place, more with |a|).  Far from 0 both are
// 0 or 1 and nothing overflows for finite a.
__device__ __forceinline__ float sigmoid(float a) {
  float e, q;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a * -LOG2E));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(1.f + e));
  return q;
}
__device__ __forceinline__ float act_value(int act, float a) {
  if (act == ERC_ACT_RELU) return a > 0.f || a != a ? a : 0.f;
  return a * (act == ERC_ACT_GELU ? 0.5f * erfcf(a * -0.7071067811865476f) : sigmoid(a));
}
__device__ __forceinline__ void act_both(int act, float a, float& value, float& slope) {
  if (act == ERC_ACT_RELU) {
    value = a > 0.f || a != a ? a : 0.f;
    slope = a > 0.f ? 1.f : 0.f;
  } else if (act == ERC_ACT_GELU) {
    const float q = 0.5f * erfcf(a * -0.7071067811865476f);
    value = a * q;
    slope = fmaf(a * expf(-0.5f * a * a), 0.3989422804014327f, q);
  } else {
    const float q = sigmoid(a);
    value = a * q;
    slope = fmaf(value, 1.f - q, q);
  }
}

// rows [first, slots) of `width` elements set to zero by all threads of the grid; `thread` of `threads`
template <class T>
__device__ __forceinline__ void zero_slots(T* out, int64_t first, int64_t slots, int64_t width, int64_t thread,
                                           int64_t threads) {
  for (int64_t i = first * width + thread; i < slots * width; i += threads) out[i] = from_f32<T>(0.f);
}

// IN or OUT for a handful of slots (expert_ffn_few.cu); rows of whole 16-byte pieces, 16-byte aligned arrays
template <class T>
erc_status ffn_few_product(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s);

// a product on the tensor cores (bfloat16 and float16 whose rows are whole 16-byte pieces); `status` (device) gets
// ERC_OK at the start of IN and DH, and ERC_ERR_TIMEOUT where a wait ran out
template <class T>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s);
template <>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<__nv_bfloat16>& p, int* status, cudaStream_t s);
template <>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<__half>& p, int* status, cudaStream_t s);

}  // namespace erc
