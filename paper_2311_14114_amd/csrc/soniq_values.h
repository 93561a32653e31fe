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
// |x / s| <= 128 the product is off by less than 2^-15, and its nearest
// integer is that of the true quotient's fp32 rounding unless it lies within
// 2^-14 of a half-integer.  There, and for scales near the ends of fp32, the
// division decides (the clamp is for subnormal scales, whose own rounding can
// exceed a step).
struct RowCoder {
  float s, rs, top;
  bool zero, fast;
  __device__ __forceinline__ RowCoder(uint32_t amax, float top_) : top(top_) {
    s = __fdiv_rn(__uint_as_float(amax), top);
    zero = !(s > 0.0f) || amax >= 0x7F800000u;
    fast = s >= 0x1p-100f && s <= 0x1p100f;
    rs = __builtin_amdgcn_rcpf(s);
  }
  // Four codes as the bytes of a word.  t = x / s + 1.5 * 2^23 holds the
  // nearest integer in its low bits: no conversion, one byte permute a pair.
  __device__ __forceinline__ uint32_t four(const float (&x)[4]) const {
    if (zero) return 0;
    constexpr float kMagic = 12582912.0f;
    uint32_t t[4];
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = __builtin_fmaf(x[i], rs, kMagic);
      far = fmaxf(far, fabsf(__builtin_fmaf(x[i], rs, kMagic - y)));  // at most a half
      t[i] = __float_as_uint(y);
    }
    if (!fast || far >= 0.5f - 0x1p-14f) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t[i] = (uint32_t)(int)fminf(fmaxf(__builtin_rintf(__fdiv_rn(x[i], s)), -top), top);
    }
    const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(t[3], t[2], 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
  }
};

// Eight neighbouring elements of a row, at any element's address.
template <int TYPE>
struct Eight {
  typedef typename Value<TYPE>::T T;
  T v[8];
  // elements from K on are zeros, and not read
  __device__ __forceinline__ void load(const T* row, int k, int K) {
    if (k + 8 <= K) {
      load(row + k);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : (T)0;
    }
  }
  __device__ __forceinline__ void load(const T* p) {
    struct __attribute__((packed, aligned(sizeof(T)))) P { T v[8]; };
    __builtin_memcpy(v, reinterpret_cast<const P*>(p), sizeof v);
  }
  // Bits of the largest |x| in fp32: their order as integers is that of the
  // values, with NaN on top; 16-bit types compare two at a time.
  __device__ __forceinline__ uint32_t amax() const {
    if constexpr (TYPE == SONIQ_F32) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
      return m;
    } else {
      typedef uint16_t u2 __attribute__((ext_vector_type(2)));
      uint32_t w[4];
      __builtin_memcpy(w, v, sizeof w);
      u2 m = {0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u2, w[i] & 0x7FFF7FFFu));
      const uint16_t x = m[0] > m[1] ? m[0] : m[1];
      return TYPE == SONIQ_BF16 ? (uint32_t)x << 16
                                : __float_as_uint((float)__builtin_bit_cast(_Float16, x));
    }
  }
  __device__ __forceinline__ uint2 codes(const RowCoder& c) const {
    float x[2][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i / 4][i % 4] = Value<TYPE>::load(v[i]);
    return make_uint2(c.four(x[0]), c.four(x[1]));
  }
  // 4-bit codes, element 2i in the low half of byte i
  __device__ __forceinline__ uint32_t nibbles(const RowCoder& c) const {
    const uint2 w = codes(c);
    const uint32_t a = w.x & 0x0F0F0F0Fu, b = w.y & 0x0F0F0F0Fu;
    return __builtin_amdgcn_perm(b | b >> 4, a | a >> 4, 0x06040200u);
  }
};

}  // namespace soniq
