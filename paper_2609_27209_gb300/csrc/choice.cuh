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

// ---- the same weights for many entries of a thread, as two sums of 32 bits
//
// For t >= -60 (smaller t are raised to it: their weights are 0 all the same) v = p 2^e is an exact
// float, hi = floor(v 2^20) and lo = round_half_up of the rest in 20 bits, so w = hi 2^20 + lo.
// floor() comes from adding 2^23 with rounding toward zero: the sum's low bits are the integer,
// and the sums of bit patterns carry a known multiple of 2^23's pattern.  Products and sums of two
// entries are issued as one packed instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2_rz(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// a * b rounded by itself: the assembler fuses a packed product with the sum that takes it (1.6 of
// 16.8 million polynomial values then differ), so the product is an fma with a -0 that it cannot see
__constant__ uint64_t minus_zeros = 0x8000000080000000ull;
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { return fma2(a, b, minus_zeros); }
__device__ __forceinline__ uint64_t fma2_rz(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

constexpr unsigned BIAS = 0x4B000000u;  // 2^23's pattern

// the polynomial of two scaled scores (|t| < 2^22), and t + 1.5 2^23, whose low bits are rint(t)
__device__ __forceinline__ void pow2_pair(float t0, float t1, float p_out[2], float r_out[2]) {
  const uint64_t t = pair(t0, t1);
  const uint64_t shifter = pair(12582912.f, 12582912.f);  // 1.5 2^23: adding it rounds to an integer
  const uint64_t r = add2(t, shifter);
  const uint64_t e = add2(r, pair(-12582912.f, -12582912.f));
  const uint64_t f = add2(t, e ^ 0x8000000080000000ull);
  uint64_t p = add2(mul2(f, pair(0.0013264727f, 0.0013264727f)), pair(0.009671513f, 0.009671513f));
  p = add2(mul2(p, f), pair(0.055507336f, 0.055507336f));
  p = add2(mul2(p, f), pair(0.24022242f, 0.24022242f));
  p = add2(mul2(p, f), pair(0.693147f, 0.693147f));
  p = add2(mul2(p, f), pair(1.f, 1.f));
  unpair(p, p_out[0], p_out[1]);
  unpair(r, r_out[0], r_out[1]);
}
// hi and lo, with their biases, of two values of 2^t
__device__ __forceinline__ void split_weights(uint64_t vv, unsigned hi[2], unsigned lo[2]) {
  const uint64_t two20 = pair(1048576.f, 1048576.f), two23 = pair(8388608.f, 8388608.f);
  const uint64_t h = fma2_rz(vv, two20, two23);
  const uint64_t rest = fma2(vv, two20, add2(two23, h ^ 0x8000000080000000ull));
  // rounded half up: half a unit is added, toward zero, before the floor
  const uint64_t l = fma2_rz(add2_rz(rest, pair(0x1p-21f, 0x1p-21f)), two20, two23);
  float a, b;
  unpair(h, a, b);
  hi[0] = __float_as_uint(a);
  hi[1] = __float_as_uint(b);
  unpair(l, a, b);
  lo[0] = __float_as_uint(a);
  lo[1] = __float_as_uint(b);
}
// weights of two scaled scores: hi and lo with their biases, and 2^t itself
__device__ __forceinline__ void weight_parts(float t0, float t1, unsigned hi[2], unsigned lo[2],
                                             float v[2]) {
  float p[2], r[2];
  pow2_pair(fmaxf(t0, -60.f), fmaxf(t1, -60.f), p, r);
  v[0] = __uint_as_float(__float_as_uint(p[0]) + (__float_as_uint(r[0]) << 23));
  v[1] = __uint_as_float(__float_as_uint(p[1]) + (__float_as_uint(r[1]) << 23));
  split_weights(pair(v[0], v[1]), hi, lo);
}
__device__ __forceinline__ unsigned long long join_parts(unsigned hi, unsigned lo) {
  return ((unsigned long long)(hi - BIAS) << 20) + (lo - BIAS);
}
// the sum of `count` weights from the sums of their parts
__device__ __forceinline__ unsigned long long join_sums(unsigned hi, unsigned lo, unsigned count) {
  return join_parts(hi - (count - 1) * BIAS, lo - (count - 1) * BIAS);
}

// 16 bytes of scores as floats; NaN becomes -inf (the maximum of a number and NaN is the number)
template <class T>
struct ScoreVec {
  static constexpr int N = 16 / sizeof(T);
};
__device__ __forceinline__ void unpack_scores(uint4 u, float* l, float) {
  l[0] = fmaxf(__uint_as_float(u.x), -INFINITY);
  l[1] = fmaxf(__uint_as_float(u.y), -INFINITY);
  l[2] = fmaxf(__uint_as_float(u.z), -INFINITY);
  l[3] = fmaxf(__uint_as_float(u.w), -INFINITY);
}
__device__ __forceinline__ void unpack_scores(uint4 u, float* l, __nv_bfloat16) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 c = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]),
                                     __nv_bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80)));
    const unsigned b = *reinterpret_cast<const unsigned*>(&c);
    l[2 * i] = __uint_as_float(b << 16);
    l[2 * i + 1] = __uint_as_float(b & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack_scores(uint4 u, float* l, __half) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 c = __hmax2(*reinterpret_cast<const __half2*>(&w[i]),
                              __half2(__ushort_as_half(0xfc00), __ushort_as_half(0xfc00)));
    const float2 f = __half22float2(c);
    l[2 * i] = f.x;
    l[2 * i + 1] = f.y;
  }
}
// the largest of 16 bytes of scores, -inf where all are masked
__device__ __forceinline__ float max_score(uint4 u, float) {
  return fmaxf(fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)),
                     fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))), -INFINITY);
}
__device__ __forceinline__ float max_score(uint4 u, __nv_bfloat16) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&u);
  const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
  return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
}
__device__ __forceinline__ float max_score(uint4 u, __half) {
  const __half2* p = reinterpret_cast<const __half2*>(&u);
  const __half2 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
  return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
}
// the same as pairs for the packed instructions
template <class T>
__device__ __forceinline__ void unpack_pairs(uint4 u, uint64_t* p) {
  float l[ScoreVec<T>::N];
  unpack_scores(u, l, T());
#pragma unroll
  for (int i = 0; i < ScoreVec<T>::N / 2; ++i) p[i] = pair(l[2 * i], l[2 * i + 1]);
}
// the pattern of -inf in each lane of a 32-bit word
template <class T>
__device__ __forceinline__ unsigned masked_word();
template <>
__device__ __forceinline__ unsigned masked_word<float>() { return 0xff800000u; }
template <>
__device__ __forceinline__ unsigned masked_word<__nv_bfloat16>() { return 0xff80ff80u; }
template <>
__device__ __forceinline__ unsigned masked_word<__half>() { return 0xfc00fc00u; }

// a row's scores as aligned 16-byte vectors: vector v holds entries v N - skew .. v N - skew + N - 1,
// those outside [0, n) read as masked.  No address outside the row is touched.
template <class T>
struct RowView {
  const T* base;  // aligned, `skew` entries before the row
  int skew;
  int n;
  int vectors;
  __device__ __forceinline__ RowView(const T* row, int64_t n_)
      : skew((int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T))), n((int)n_) {
    base = row - skew;
    vectors = (skew + n + ScoreVec<T>::N - 1) / ScoreVec<T>::N;
  }
  // vectors that lie wholly inside the row: (v > 0 or no skew) and v < whole()
  __device__ __forceinline__ int whole() const { return (skew + n) / ScoreVec<T>::N; }
  __device__ __forceinline__ uint4 inner(int v) const {
    return __ldg(reinterpret_cast<const uint4*>(base) + v);
  }
  __device__ __forceinline__ uint4 fetch(int v) const {
    const int first = v * ScoreVec<T>::N - skew;
    return first >= 0 && first + ScoreVec<T>::N <= n ? inner(v) : edge(base, skew, n, first);
  }
  static __device__ __noinline__ uint4 edge(const T* base, int skew, int n, int first) {
    constexpr int N = ScoreVec<T>::N;
    union {
      uint4 u;
      T t[N];
      unsigned w[4];
    } x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.w[i] = masked_word<T>();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (first + i >= 0 && first + i < n) x.t[i] = base[skew + first + i];
    return x.u;
  }
};

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
