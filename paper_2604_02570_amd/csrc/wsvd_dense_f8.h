// 8-bit pages of dense layers: codes and scales as the kernels see them.
//
// A block is 16 consecutive rows of one kv head, d bytes of E4M3 codes a row and one scale 2^e for its keys and one for its values,
// held as the byte e + 127.  A page holds page_rows / 16 blocks of every kv head.  The bytes of a block lie as the matrix cores take them:
//   keys    [d / 16][16 rows][16 dims]: lane L of a wave asks for the 16 bytes of row L % 16 that it has in the score product
//   values  [d / 64][4 groups of 4 rows][64 dims][4 rows]: a dword is what a lane has of 4 rows in the value product
// so that whole waves ask for 1 KB in one piece, and operands are made by conversion alone: a scale that is a power of two goes
// into the conversion of two codes to two 16-bit numbers, and leaves them exact.
#pragma once
#include "wsvd_dense.h"

constexpr int kF8Rows = 16, kF8Bias = 127, kF8Least = -100;
// The codes are limited where the scale is so large that the ones above would stand for numbers past the type (256 * 2^8 in f16).
template <class T> struct F8Top { static constexpr int exponent = 120; };
template <> struct F8Top<DenseF16> { static constexpr int exponent = 8; };

// The least e with most <= 448 * 2^e (448 is 1.75 * 2^8: one mantissa above 0.75 more makes the exponent's carry), at least kF8Least.
WSVD_DEV int f8_exponent(float most) { return max((int)((__float_as_uint(most) + 0x1FFFFFu) >> 23) - 135, kF8Least); }
WSVD_DEV float f8_power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // 2^e, e in -126 .. 127
WSVD_DEV bool f8_finite(float x) { return __builtin_fabsf(x) < INFINITY; }
// A number over its scale as what the conversion takes: none for those that are infinite or none.
WSVD_DEV float f8_scaled(float x, float inverse, float top) {
  return f8_finite(x) ? __builtin_amdgcn_fmed3f(x * inverse, -top, top) : __builtin_nanf("");
}
// The larger of a magnitude and those of two numbers, infinite ones and none left out.
template <class T>
WSVD_DEV float f8_most(float most, uint32_t x) {
  const float a = __builtin_fabsf(dense_low<T>(x)), b = __builtin_fabsf(dense_high<T>(x));
  return fmaxf(most, fmaxf(f8_finite(a) ? a : 0.f, f8_finite(b) ? b : 0.f));
}
template <class T>
WSVD_DEV float f8_top(int e) { return e >= F8Top<T>::exponent ? 240.f : 448.f; }
WSVD_DEV uint32_t f8_codes(float a, float b, float c, float d) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}
// The first n bytes of a dword, all for 4 and more, none for 0 and less.
WSVD_DEV uint32_t f8_bytes(int n) { return n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1u; }
// Codes under a scale that is `by` times smaller than the one they had (by = 2^-n): rounded to nearest even, exact unless they become subnormal.
WSVD_DEV uint32_t f8_moved(uint32_t codes, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return f8_codes(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}
// Two codes times a power of two as two numbers of the type, the first in the low half.
template <class T, bool HIGH>
WSVD_DEV int f8_pair(uint32_t codes, float scale) {
  if constexpr (__is_same(T, DenseBf16)) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
  else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HIGH));
}
// Where a block lies: its number among the blocks of the pools, page * Hkv * (page_rows / 16) + ...
WSVD_DEV uint64_t f8_block(int page, int granule, int pg, int kv, int Hkv, int page_rows) { return dense_pool_row(page, granule, pg, kv, Hkv, page_rows) >> 4; }
