// The 4-bit cache rows that several sources write or read (gfx950).
//
// A row x of D values is D / 32 blocks of 32 values, each 32 e2m1 codes (0, 0.5, 1,
// 1.5, 2, 3, 4, 6 and a sign; two in a byte, the first in its low half) and one
// exponent byte e, and stands for code * 2^(e - 127); e = 255 stands for 32 NaN.
// e is the smallest number in [1, 254] with max |x_i| <= 7 * 2^(e - 127): 7 is where
// half a step past the largest code ends, so a value is off by at most half the
// step at its size, and the block's other values keep the finest steps that allow
// this.  (With 6 for 7 the largest value of a block, where it lies between, is
// halved instead of rounded down, and every other value's step doubles.)
// Both directions are one instruction for two values, and an operand's power of
// two rides along: the conversion takes a scale's exponent field, 255 as NaN.
#pragma once

#include "q8.h"

namespace pvlm {

// Padded or paged, as an 8-bit cache (see Q8Cache); a row is D / 2 bytes of codes
// and D / 32 of exponents.
typedef Q8Cache Q4Cache;
__device__ __forceinline__ int64_t q4_row(const Q4Cache& c, int l, int B, int b, int Hkv, int g, int64_t row) {
  return q8_row(c, l, B, b, Hkv, g, row);
}

// The exponent byte of a block whose largest magnitude is `top` (no NaN): 7 =
// 1.75 * 2^2; 255 for an infinity.
__device__ __forceinline__ int q4_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  if (u >= 0x7f800000u) return 255;
  const int e = (int)(u >> 23) - 2 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 1 ? 1 : e;
}

// |x|, an infinity for NaN
__device__ __forceinline__ float abs_or_inf(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return __uint_as_float(u < 0x7f800000u ? u : 0x7f800000u);
}

// Eight codes of x * 2^(127 - e), nearest, ties to the even code, at most 6 (0 for
// e = 255).  Not the instruction's own scale: 2^(e - 127) of a small e would be
// subnormal in it.
__device__ __forceinline__ uint32_t e2m1x8(const float* x, int e) {
  if (e == 255) return 0u;
  const float f = q8_scale(e);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0] * f, x[1] * f, 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * f, x[3] * f, 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * f, x[5] * f, 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * f, x[7] * f, 1.f, 3);
}

// A lane's 8 values of a row; its block's other values are with the next three of
// each aligned four lanes.
__device__ __forceinline__ uint32_t q4_encode(const float (&x)[8], int& e) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, abs_or_inf(x[i]));
  top = fmaxf(top, lane_xor1(top));
  top = fmaxf(top, lane_xor2(top));
  e = q4_exponent(top);
  return e2m1x8(x, e);
}

__device__ __forceinline__ void bf16x8_to_f32(uint4 u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// What every call checks of a 4-bit cache's pointers and capacity: vectors of up to
// 16 bytes of codes, 4 bytes of exponents, blocks of 32 rows that a read may take whole.
inline pvlm_status check_q4(const void* kc, const void* ke, const void* vc, const void* ve, int64_t n_cap) {
  return check_q8(kc, ke, vc, ve, n_cap);
}

}  // namespace pvlm
