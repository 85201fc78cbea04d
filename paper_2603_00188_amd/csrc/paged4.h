// Rows of a 4-bit pool (STLITE_KV4 in include/stlite_paged.h) on the device: 128 values
// as four blocks of 32 codes (a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6) and a scale
// byte each, the scale being 2^(byte - 127) and NaN for 255.  gfx950 converts pairs of
// codes to 16 bits and back under such a scale in one instruction at the rate of an add
// (to codes: half of it), rounding to nearest, ties to the even code, and stopping at 6.
#pragma once

#include "paged.h"

namespace stlite {

constexpr int32_t kCodes4 = 64;  // bytes of a row's codes
constexpr int32_t kRow4 = 68;    // and with its scales

// First byte of page `page` of a unit: page_size rows of codes, then of scales.
__device__ inline int64_t page4(const PagedDev& c, int32_t unit, int32_t page) { return page_row(c, unit, page) * kRow4; }

// The float of a scale byte.
__device__ inline float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

template <typename T>
struct Four;
template <>
struct Four<__bf16> {
  typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
  // Least and greatest byte of a scale: 2^-120 and 2^125, so that every value is a
  // normal finite bf16.
  static constexpr int32_t kLeast = 7, kMost = 252;
  // Byte SEL of `codes` as two values.
  template <int SEL>
  static __device__ uint32_t values(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
  }
  template <int SEL>
  static __device__ uint32_t codes(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(pair_t, pair), scale, SEL);
  }
  // fp32 bits of a magnitude's bits.
  static __device__ uint32_t wide(uint32_t bits) { return bits << 16; }
};
template <>
struct Four<_Float16> {
  typedef _Float16 pair_t __attribute__((ext_vector_type(2)));
  static constexpr int32_t kLeast = 113, kMost = 140;  // 2^-14 and 2^13 (6 2^14 is no half)
  template <int SEL>
  static __device__ uint32_t values(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
  }
  template <int SEL>
  static __device__ uint32_t codes(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(pair_t, pair), scale, SEL);
  }
  static __device__ uint32_t wide(uint32_t bits) { return __float_as_uint(float(__builtin_bit_cast(_Float16, uint16_t(bits)))); }
};

// The scale byte of a block whose greatest magnitude has the fp32 bits `top`: the least
// power of two with top <= 7 of it.  (From 6 to 7 of it the greatest value is off by as
// much as it would be under twice the scale, and the others by less.)
template <typename T>
__device__ inline uint32_t scale_byte(uint32_t top) {
  const int32_t e = int32_t((top + 0x1fffffu) >> 23) - 2;
  return top >= 0x7f800000u ? 255u : uint32_t(min(max(e, Four<T>::kLeast), Four<T>::kMost));
}

// Eight values of a row, in 16 bits, as codes, element i in bits 4 i (none for a scale of 255).
template <typename T>
__device__ inline uint32_t codes_of(const uint32_t (&w)[4], uint32_t byte) {
  const float s = scale_of(byte);
  uint32_t c = Four<T>::template codes<0>(0u, w[0], s);
  c = Four<T>::template codes<1>(c, w[1], s);
  c = Four<T>::template codes<2>(c, w[2], s);
  c = Four<T>::template codes<3>(c, w[3], s);
  return byte == 255u ? 0u : c;
}
// The same from fp32.
__device__ inline uint32_t codes_of(const float (&x)[8], uint32_t byte) {
  const float s = scale_of(byte);
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  return byte == 255u ? 0u : c;
}

// The greatest magnitude of eight 16-bit values, as 16 bits.
__device__ inline uint32_t top_of(const uint32_t (&w)[4]) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  u16x2_t m = __builtin_bit_cast(u16x2_t, w[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, w[i] & 0x7fff7fffu));
  return max(uint32_t(m[0]), uint32_t(m[1]));
}

// Eight codes as values.
template <typename T>
__device__ inline void values_of(uint32_t codes, float scale, uint32_t (&w)[4]) {
  w[0] = Four<T>::template values<0>(codes, scale);
  w[1] = Four<T>::template values<1>(codes, scale);
  w[2] = Four<T>::template values<2>(codes, scale);
  w[3] = Four<T>::template values<3>(codes, scale);
}

// Eight codes without those whose values are not finite under a scale byte above kMost (any
// other: all of them stay): 4 and 6 one above it, from 2 on two above, from 1 on, from 1/2 on;
// of 255 none stays.
template <typename T>
__device__ inline uint32_t finite_codes(uint32_t codes, uint32_t byte) {
  const uint32_t b0 = codes, b1 = codes >> 1, b2 = codes >> 2;
  uint32_t odd = byte > uint32_t(Four<T>::kMost) ? b2 & b1 : 0u;  // (bit 4 i: code i)
  if (byte > uint32_t(Four<T>::kMost) + 1) odd = b2;
  if (Four<T>::kMost < 252 && byte > uint32_t(Four<T>::kMost) + 2) odd = byte > uint32_t(Four<T>::kMost) + 3 ? b2 | b1 | b0 : b2 | b1;
  if (byte == 255u) odd = ~0u;
  return codes & ~((odd & 0x11111111u) * 15u);
}

}  // namespace stlite
