// choice.cuh -- what the row-wise choice operators share: loads of the three score types and the
// fixed-point exponential that makes their whole-number results the same on every machine.
//
// 2^t for t <= 0 is p(f) 2^e with e = rint(t), f = t - e in [-1/2, 1/2] (exact) and p a degree-5
// polynomial through p(0) = 1, fitted to 2^f for the smallest relative error (9.1e-8; 1.9e-7 with
// the rounding of its float32 evaluation).  Each product and sum is rounded by itself, never fused,
// so any float32 arithmetic reproduces its bits.  A weight is round(p 2^(e+40)), half up, as an
// integer: sums of weights are exact and do not depend on their order.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "erc_internal.cuh"

namespace erc {

constexpr float LOG2E = 1.4426950408889634f;

template <class T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// a score as the operators see it: NaN counts as masked, and -0 equals +0
__device__ __forceinline__ float clean_score(float v) { return v != v ? -INFINITY : __fadd_rn(v, 0.f); }

__device__ __forceinline__ float pow2_poly(float f) {
  float p = __fadd_rn(__fmul_rn(f, 0.0013264727f), 0.009671513f);
  p = __fadd_rn(__fmul_rn(p, f), 0.055507336f);
  p = __fadd_rn(__fmul_rn(p, f), 0.24022242f);
  p = __fadd_rn(__fmul_rn(p, f), 0.693147f);
  return __fadd_rn(__fmul_rn(p, f), 1.f);
}

// round(2^t 2^40) for t <= 0; 0 below 2^-41.5 and for NaN
__device__ __forceinline__ unsigned long long fixed_weight(float t) {
  if (!(t > -41.5f)) return 0ull;
  const float e = rintf(t);
  const float p = pow2_poly(__fsub_rn(t, e));
  const unsigned long long m = (unsigned)__fmul_rn(p, 16777216.f);  // exact: p >= 1/2
  return (((m << 17) >> (int)(-e)) + 1) >> 1;
}

// 2^t as a float, 0 where rint(t) < least (>= -126) and for NaN
__device__ __forceinline__ float pow2_float(float t, float least) {
  const float e = rintf(t);
  if (!(e >= least)) return 0.f;
  return __fmul_rn(pow2_poly(__fsub_rn(t, e)), __int_as_float(((int)e + 127) << 23));
}

// (l - max) scale for l <= max, 0 at the maximum whatever the scale
__device__ __forceinline__ float below_max(float l, float max, float scale) {
  return l == max ? 0.f : __fmul_rn(__fsub_rn(l, max), scale);
}

// floats in an order that unsigned comparison keeps (larger float, larger key; never 0 for a number)
__device__ __forceinline__ unsigned order_key(float v) {
  const unsigned b = __float_as_uint(v);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(unsigned k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

inline int type_bytes(int32_t type) { return type == ERC_F32 ? 4 : 2; }

// calls f with a value of the C++ type behind an erc_type (checked by the caller)
template <class F>
erc_status with_type(int32_t type, F&& f) {
  switch (type) {
    case ERC_F32: return f(float());
    case ERC_BF16: return f(__nv_bfloat16());
    default: return f(__half());
  }
}

}  // namespace erc
