// Microscaled 4-bit floating point (MXFP4) in device code: e2m1 codes, two to a
// byte (low nibble first), and one e8m0 scale byte s per 32 elements:
//     value = code * 2^(s - 127),   code in +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.
// s = 255 makes every element of its block NaN.  A value has two significant
// bits, so it is exact in bf16 (past bf16's range it is an infinity), and a
// product with 4-bit operands is the bf16 MFMA on the converted values: no
// rounding but that of the fp32 accumulation.
#pragma once
#include "common.h"

namespace al {

// The conversions take the scale as an fp32 number whose exponent field is the
// scale byte (checked for every scale byte and code on MI355X, 0 and 255 too).
__device__ __forceinline__ float mx4_scale(unsigned s) { return __uint_as_float(s << 23); }

// Eight elements: the nibbles of c, lowest first.
__device__ __forceinline__ bf16x8 mx4_bf16x8(unsigned c, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
  i32x4 r = {__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), __builtin_bit_cast(int, d),
             __builtin_bit_cast(int, e)};
  return __builtin_bit_cast(bf16x8, r);
}

// Quantises a block of 32 elements held by four neighbouring lanes (lane 4 i + j
// elements 8 j .. 8 j + 7, x their bf16 bits): returns the lane's eight codes and
// the block's scale byte.  The scale's exponent is that of the largest
// magnitude less 2, so that magnitude is in [4, 8) scales (6 at most is kept);
// codes are rounded to nearest, ties to even, by the conversion itself.  A block
// with an infinity or NaN gets scale byte 255 and zero codes.
__device__ __forceinline__ unsigned mx4_quantize8(i32x4 x, unsigned& s) {
  // Magnitudes order as their bits do.
  unsigned hi = 0, lo = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi = max(hi, (unsigned)x[i] & 0x7FFF0000u);
    lo = max(lo, (unsigned)x[i] & 0x7FFFu);
  }
  unsigned m = max(hi >> 16, lo);
  m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));   // lane ^ 2
  const unsigned e = m >> 7;
  if (e == 255) {
    s = 255;
    return 0;
  }
  s = e > 2 ? e - 2 : 0;
  const float scale = mx4_scale(s);
  const int x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];   // (a bit cast of x[i] itself would take element 0)
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), scale, 3);
  return c;
}

}  // namespace al
