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

// looks at a barrier before a wait gives up, and how many nanoseconds a look may sleep: one that is told to give up
// early does not sleep
struct TcPatience {
  unsigned polls = 0x7fffffffu, nap = 1000000u;
  TcPatience() = default;
  __host__ __device__ explicit TcPatience(unsigned limit) { if (limit) polls = limit, nap = 0; }
};

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
  // DWIN and DWOUT: the slots of an expert in `splits` parts, whose sums go to partial [splits][experts][rows][columns]
  int splits;
  float* partial;
  // on the tensor cores: how long a wait lasts, and which blocks of IN or DH gave up
  TcPatience patience;
  int* lost;
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
// the slots of part `s` of an expert's [lo, hi)
__device__ __forceinline__ SlotRange split_range(SlotRange r, int s, int splits) {
  if (splits == 1) return r;
  const int64_t each = ((r.hi - r.lo + splits - 1) / splits + 63) & ~int64_t(63);
  const int64_t lo = r.lo + s * each, hi = lo + each;
  return {lo < r.hi ? lo : r.hi, hi < r.hi ? hi : r.hi};
}

__device__ __forceinline__ int64_t slots_used(const int64_t* offsets, int experts, int64_t slots) {
  const int64_t v = __ldg(offsets + experts);
  return v < 0 ? 0 : v > slots ? slots : v;
}


// act(a), and act'(a).  The sigmoid takes the hardware's 2^x and 1 / x (a few units in the last place, more with |a|).  The
// normal distribution function of -|a| is e^(-a^2 / 2) G(1 / (1 + 0.34 |a|)), G a polynomial without a constant term
// fitted to e^(a^2 / 2) erfc(|a| / sqrt 2) / 2 for the smallest relative error on [0, 14.5] (4e-8; 4e-7 with the rounding
// of its float32 evaluation), so its lower tail keeps its relative accuracy.  Far from 0 both functions are 0 or 1 and
// nothing overflows for finite a.
__device__ __forceinline__ float exp2_hw(float t) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}
__device__ __forceinline__ float recip_hw(float t) {
  float q;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(t));
  return q;
}
__device__ __forceinline__ float sigmoid(float a) { return recip_hw(1.f + exp2_hw(a * -LOG2E)); }

constexpr float HALF_LOG2E = 0.72134752f;
constexpr float TAIL_STEP = 0.34f;
__host__ __device__ constexpr float tail_coef(int i) {
  constexpr float c[9] = {0.135621578f, 0.136092216f, 0.115351841f, 0.114712983f, 
                          -0.0431046113f, 0.199714825f, -0.270868301f, 0.138355583f, -0.0258760974f};
  return c[i];
}
// the normal distribution function of a, and e^(-a^2 / 2)
__device__ __forceinline__ float normal_below(float a, float& e) {
  const float t = recip_hw(fmaf(TAIL_STEP, fabsf(a), 1.f));
  float g = tail_coef(8);
#pragma unroll
  for (int i = 7; i >= 0; --i) g = fmaf(g, t, tail_coef(i));
  e = exp2_hw(a * a * -HALF_LOG2E);
  const float q = g * t * e;
  return a < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float act_value(int act, float a) {
  if (act == ERC_ACT_RELU) return a > 0.f || a != a ? a : 0.f;
  float e;
  return a * (act == ERC_ACT_GELU ? normal_below(a, e) : sigmoid(a));
}
__device__ __forceinline__ void act_both(int act, float a, float& value, float& slope) {
  if (act == ERC_ACT_RELU) {
    value = a > 0.f || a != a ? a : 0.f;
    slope = a > 0.f ? 1.f : 0.f;
  } else if (act == ERC_ACT_GELU) {
    float e;
    const float q = normal_below(a, e);
    value = a * q;
    slope = fmaf(a * e, 0.3989422804014327f, q);
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

// blocks of every product on the tensor cores
inline int tc_blocks() { return sm_count() / 2 * 2; }

// IN or OUT for a handful of slots (expert_ffn_few.cu); rows of whole 16-byte pieces, 16-byte aligned arrays
template <class T>
erc_status ffn_few_product(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s);

// a product on the tensor cores (bfloat16 and float16 whose rows are whole 16-byte pieces); `status` (device) gets
// ERC_OK at the start of IN and DH, and ERC_ERR_TIMEOUT where a wait ran out: IN and DH leave word in `lost`, which the
// products after them pass on, so that none can undo it
template <class T>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<T>& p, int* status, cudaStream_t s);
template <>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<__nv_bfloat16>& p, int* status, cudaStream_t s);
template <>
erc_status ffn_tc_product(FfnProduct which, const FfnArgs<__half>& p, int* status, cudaStream_t s);

}  // namespace erc
