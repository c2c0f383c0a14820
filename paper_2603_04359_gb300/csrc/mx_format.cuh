// The microscaled 4-bit format (MXFP4 of the OCP Microscaling Formats specification, v1.0) as the kernels read and
// write it: a row of d values is d / 2 bytes of E2M1 codes (value 2j in the low nibble of byte j) and one scale byte
// per 32 values, 2^(b - 127), 255 for NaN.  The scale bytes of a row take mx_pitch(d) bytes, a multiple of 16 (the unit
// of a tensor copy), of which the bytes past d / 32 are zero.
#pragma once
#include "common.cuh"

namespace cat {

constexpr int64_t kMxMaxExperts = 1024;

__host__ __device__ constexpr int64_t mx_pitch(int64_t d) { return (d + 511) / 512 * 16; }

// The scale byte of a block whose largest magnitude has these bits: the power of two two binades below the largest
// magnitude's own, so that it lands in [4, 8) and at most its part above 6, the largest E2M1 value, saturates.  A block
// with an infinity or a NaN (bits of 0x7f800000 and more) has the NaN scale.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255u;
  const int b = (int)(amax_bits >> 23) - 2;
  return b > 0 ? (uint32_t)b : 0u;
}
// 2^(127 - b), exact: what a value is multiplied by before it is rounded (b <= 252 as made above).
__device__ __forceinline__ float mx_inverse_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// 2^(b - 127), exact; NaN for 255.
__device__ __forceinline__ float mx_scale(uint32_t b) {
  return __uint_as_float(b == 255u ? 0x7FFFFFFFu : b == 0u ? 0x00400000u : b << 23);
}

// Eight values (already divided by the scale) to E2M1, nearest with ties to even, magnitudes over 6 to 6: v[0] in the
// low nibble of the first byte.
__device__ __forceinline__ uint32_t mx_pack8(const float (&v)[8]) {
  uint32_t w;
  asm("{ .reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d}; }"
      : "=r"(w)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return w;
}

// The value of a code: bit 3 the sign, bits 0 to 2 the magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6.
__device__ __forceinline__ float mx_code_value(uint32_t c) {
  const uint32_t m = c & 7u;
  // exponent field and one mantissa bit of a float: m >= 2 is 2^(m/2 - 1) (1 + (m & 1) / 2); 1 is 0.5; 0 is 0
  const uint32_t bits = m >= 2u ? ((126u + (m >> 1)) << 23) | ((m & 1u) << 22) : m ? 0x3F000000u : 0u;
  return __uint_as_float(bits | ((c & 8u) << 28));
}

}  // namespace cat
