// fp8.h -- e4m3 codes with power-of-two scales.
//
// A scale is kept as its exponent plus 127 in a byte, so that 2^e is the float
// of the bits byte << 23, but for byte 0, 2^-127, which is subnormal (and what a zeroed pool
// holds).  The bytes written here are at least kMinScale, where the least code is 2^-9 2^-117,
// a normal number, so that a code times a scale, of four significant bits, is exact in bf16 and
// fp32.  Any scale is exact in fp32; bytes below 3 leave codes whose last bits are below
// 2^-133, where bf16 ends, and which round there to nearest even.
#pragma once

#include "device.h"

namespace hyb {

constexpr int kMinScale = 10;  // 2^-117

// (Positive for every number: -infinity times it, a hidden score, stays one.)  NaN for byte 255,
// as in the conversions, where an infinity would drop the tokens whose scores it makes negative.
__device__ inline float scale_of(int byte) {
  return __builtin_bit_cast(float, max(byte << 23 | (byte + 1) >> 8 << 22, 0x400000));
}

// The byte of the least e with m <= 448 2^e, for the bits of a finite m >= 0.
// 448 is 1.75 2^8: the mantissa's part above 1.75 carries into the exponent.
__device__ inline int scale_byte(int bits) { return max(((bits + 0x1fffff) >> 23) - 8, kMinScale); }

// Four codes (a dword) as floats, times f; eight as a bf16 operand, times 2^e = f (the
// conversion takes f's exponent).
__device__ inline f32x4 fp8_f32(uint32_t c, float f) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4{a[0] * f, a[1] * f, b[0] * f, b[1] * f};
}
__device__ inline bf16x8 fp8_bf16(uint32_t c0, uint32_t c1, float f) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// x f as codes, rounded to nearest even; NaN where x is not finite (an infinity has no
// code).  |x| f is at most 448 where f is the block's.
__device__ inline uint32_t fp8_codes(float x0, float x1, float x2, float x3, float f) {
  auto y = [f](float x) { return __builtin_fabsf(x) < INFINITY ? x * f : __builtin_nanf(""); };
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(y(x0), y(x1), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y(x2), y(x3), c, true);
}

}  // namespace hyb
