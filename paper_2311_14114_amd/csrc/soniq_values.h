// Values of the types the serving kernels read and write, and the codec's
// arithmetic on them.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

#include "soniq.h"

namespace soniq {

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ __forceinline__ uint16_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest even, NaN stays NaN
}

template <int TYPE>
struct Value;
template <>
struct Value<SONIQ_F32> {
  typedef float T;
  static __device__ __forceinline__ float load(T v) { return v; }
  static __device__ __forceinline__ T store(float x) { return x; }
};
template <>
struct Value<SONIQ_BF16> {
  typedef uint16_t T;
  static __device__ __forceinline__ float load(T v) { return bf16_value(v); }
  static __device__ __forceinline__ T store(float x) { return bf16_bits(x); }
};
template <>
struct Value<SONIQ_F16> {
  typedef _Float16 T;
  static __device__ __forceinline__ float load(T v) { return (float)v; }
  static __device__ __forceinline__ T store(float x) {
    // x is a rounded fp32 value: without this a product and its conversion
    // become one instruction that rounds once, here and there
    asm("" : "+v"(x));
    return (_Float16)x;
  }
};

// The symmetric codec of a row whose largest |x| has the bits `amax` (as an
// unsigned integer, so that a NaN or an infinity is the largest):
// s = amax / top, code = rint(x / s), both divisions IEEE fp32.  A scale of 0,
// infinity or NaN gives codes 0.
//
// The quotient comes from a reciprocal: v_rcp_f32 is good to one ulp, so for
// |x / s| <= 128 the product is off by less than 2^-15, and rint of it is
// rint of the true quotient's fp32 rounding unless it lies within 2^-14 of a
// half-integer.  There, and for scales near the ends of fp32, the division
// decides.  The clamp is for subnormal scales, whose own rounding can exceed
// a step.
struct RowCoder {
  float s, rs, top;
  bool zero, fast;
  __device__ __forceinline__ RowCoder(uint32_t amax, float top_) : top(top_) {
    s = __fdiv_rn(__uint_as_float(amax), top);
    zero = !(s > 0.0f) || amax >= 0x7F800000u;
    fast = s >= 0x1p-100f && s <= 0x1p100f;
    rs = __builtin_amdgcn_rcpf(s);
  }
  template <int N>
  __device__ __forceinline__ void code(const float (&x)[N], int (&q)[N]) const {
    float t[N], far = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = x[i] * rs;
      t[i] = __builtin_rintf(e);
      far = fmaxf(far, fabsf(e - t[i]));  // at most a half
    }
    if (!fast || far >= 0.5f - 0x1p-14f) {
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = fminf(fmaxf(__builtin_rintf(__fdiv_rn(x[i], s)), -top), top);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = zero ? 0 : (int)t[i];
  }
};

}  // namespace soniq
