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
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);  // NaN stays NaN
  return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
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
  static __device__ __forceinline__ T store(float x) { return (_Float16)x; }
};

// N elements at any element-aligned address, in the widest loads and stores
// there are (the hardware takes them at any alignment).
template <class T, int N>
struct alignas(1) Pack {
  T v[N];
} __attribute__((packed));

// The symmetric codec of a row whose largest |x| has the bits `amax` (as an
// unsigned integer, so that a NaN or an infinity is the largest): its scale,
// and its codes' range.  A scale of 0, infinity or NaN gives codes 0.
struct RowCodec {
  float s;
  bool zero;
  float top;
};
__device__ __forceinline__ RowCodec row_codec(uint32_t amax, float top) {
  RowCodec r;
  r.s = __fdiv_rn(__uint_as_float(amax), top);
  r.zero = !(r.s > 0.0f) || amax >= 0x7F800000u;
  r.top = top;
  return r;
}
__device__ __forceinline__ int row_code(const RowCodec& r, float x) {
  if (r.zero) return 0;
  // the clamp is for subnormal scales, whose own rounding can exceed a step
  return (int)fminf(fmaxf(__builtin_rintf(__fdiv_rn(x, r.s)), -r.top), r.top);
}

}  // namespace soniq
