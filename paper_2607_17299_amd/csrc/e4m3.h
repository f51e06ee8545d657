// Eight-bit floats (OCP e4m3, no infinities) with power-of-two scales.
//
// A block of numbers x has the scale 2^e, e the smallest integer with
// max |x| <= 448 2^e, at least -117: the codes then stand for normal bf16 numbers
// (the smallest is 2^-9 2^e), so code * 2^e is exact in bf16.  Multiplying by a power
// of two is exact as well: a block's codes are the one rounding (to nearest even) of
// its numbers, whoever writes them.
#pragma once

#include "common.h"

constexpr int kMinExp8 = -117, kNanCode8 = 0x7f;

// e for a block's largest magnitude (finite, >= 0): a = m 2^p with 1 <= m < 2, and
// 448 = 1.75 2^8.  A subnormal a has p below the range and takes the least e.
WAR_DEV int block_exp8(float a) {
  const uint32_t u = __float_as_uint(a);
  const int p = (int)(u >> 23) - 127;
  return max(p - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), kMinExp8);
}
WAR_DEV float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// codes of two numbers already divided by their scale, in bits 0..15
WAR_DEV uint32_t to_e4m3x2(float a, float b) { return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu; }
WAR_DEV uint32_t to_e4m3x4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// bf16 numbers of codes 0, 1 (HI: 2, 3) of a word, times a power of two
template <bool HI>
WAR_DEV uint32_t from_e4m3x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// eight numbers of one scale
WAR_DEV uint4 from_e4m3x8(uint32_t w0, uint32_t w1, float scale) {
  return make_uint4(from_e4m3x2<false>(w0, scale), from_e4m3x2<true>(w0, scale), from_e4m3x2<false>(w1, scale),
                    from_e4m3x2<true>(w1, scale));
}
// code I of a word times a power of two
template <int I>
WAR_DEV float from_e4m3(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_f32_fp8((int)w, scale, I);
}
// the scale of byte I of a word of scale bytes (byte 0: 0)
template <int I>
WAR_DEV float scale_of(uint32_t w) {
  return __uint_as_float(((w >> (8 * I)) & 0xff) << 23);
}
