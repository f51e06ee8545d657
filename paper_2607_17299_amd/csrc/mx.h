// Microscaled numbers: 32 neighbours of a row share a power-of-two scale 2^e, kept as
// the byte e + 127; their codes are e4m3 (a byte) or e2m1 (4 bits, the even column in the
// low ones).  e is the smallest integer with max |x| <= top 2^e (448 or 6), at least
// -117, so dividing by the scale is exact and a code is the one rounding (nearest, ties
// to even) of its number.  A block with a number that is not finite has the scale byte
// 255, which stands for NaN.
#pragma once

#include "e4m3.h"
#include "kernels.h"

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kMxE4M3 = 0, kMxE2M1 = 1;  // war.h's WAR_MX_* less WAR_MX_E4M3
constexpr int kNanScale = 255;

// e for a block's largest magnitude (finite, >= 0): 448 = 1.75 2^8, 6 = 1.5 2^2
template <int FMT>
WAR_DEV int mx_exp(float a) {
  if constexpr (FMT == kMxE4M3) return block_exp8(a);
  const uint32_t u = __float_as_uint(a);
  return max((int)(u >> 23) - 127 - 2 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0), kMinExp8);
}
// e2m1 codes of eight numbers already divided by their scale
WAR_DEV uint32_t to_e2m1x8(const float (&y)[8]) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
}
// The largest (and whether any is set) of the four neighbouring lanes that hold a block.
WAR_DEV float quad_max(float v) {
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0xb1, 0xf, 0xf, true)));
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x4e, 0xf, 0xf, true)));
}
// Eight numbers of a block whose others are in the three neighbouring lanes (lanes
// 4 i .. 4 i + 3): their codes to `codes`, the scale byte by the block's first lane.  A
// number that is not finite makes x * 0 NaN, which carries it into the maximum as infinity.
template <int FMT>
WAR_DEV void mx_store8(const float (&x)[8], uint8_t* codes, uint8_t* scale, bool first) {
  float top = 0.f, odd = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = fmaxf(top, fabsf(x[i]));
    odd = fmaf(x[i], 0.f, odd);
  }
  top = quad_max(odd == 0.f ? top : INFINITY);
  const bool bad = top == INFINITY;
  const int e = mx_exp<FMT>(bad ? 0.f : top);
  const float f = exp2_int(-e);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * f;
  if constexpr (FMT == kMxE4M3) {
    const uint2 c = make_uint2(to_e4m3x4(y[0], y[1], y[2], y[3]), to_e4m3x4(y[4], y[5], y[6], y[7]));
    *reinterpret_cast<uint2*>(codes) = bad ? make_uint2(0, 0) : c;
  } else {
    const uint32_t c = to_e2m1x8(y);
    *reinterpret_cast<uint32_t*>(codes) = bad ? 0 : c;
  }
  if (first) *scale = bad ? kNanScale : (uint8_t)(e + 127);
}
// 2^(byte - 127) of a scale byte (0: the subnormal 2^-127; 255: NaN)
WAR_DEV float mx_scale(int b) { return b == kNanScale ? __builtin_nanf("") : __uint_as_float(b ? (uint32_t)b << 23 : 0x400000u); }
