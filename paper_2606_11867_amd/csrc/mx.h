// Microscaled 4-bit floats on the device: blocks of 32 elements with a
// power-of-two scale (include/foremoe.h).
#pragma once

#include "common.h"

namespace foremoe {

constexpr int kMxBlock = FOREMOE_MX_BLOCK;

// Scale byte of a block from the bits of its largest magnitude: the least e
// with amax < 7 * 2^e, from the exponent and whether the significand reaches
// 1.75. A NaN or infinity has the byte 255.
__device__ __forceinline__ uint32_t mx_scale_of(uint32_t amax_bits) {
  const int e = (int)((amax_bits + 0x200000u) >> 23) - 2;  // e + 127
  const int c = e < 0 ? 0 : (e > 252 ? 252 : e);
  return amax_bits >= 0x7f800000u ? 255u : (uint32_t)c;
}

// 2^-e, exact for every e that mx_scale_of gives (NaN blocks: their elements
// are not looked at).
__device__ __forceinline__ float mx_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// Codes of a and b (over their scale) in the low byte and the next. The
// instruction rounds to nearest even and saturates at 6.
template <int BYTE>
__device__ __forceinline__ uint32_t mx_put2(uint32_t word, float a, float b) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, 1.0f, BYTE);
}

__device__ __forceinline__ uint32_t mx_put8(const float* y) {
  uint32_t w = mx_put2<0>(0u, y[0], y[1]);
  w = mx_put2<1>(w, y[2], y[3]);
  w = mx_put2<2>(w, y[4], y[5]);
  return mx_put2<3>(w, y[6], y[7]);
}

// A scale byte as the conversions and the matrix instructions take it: the
// exponent bits of a float (0: 2^-127; 255: NaN).
__device__ __forceinline__ float mx_scale_operand(uint32_t scale) { return __uint_as_float(scale << 23); }

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The two values of one byte of a word.
template <int BYTE>
__device__ __forceinline__ f32x2_t mx_get2(uint32_t word, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, BYTE);
}
template <int BYTE>
__device__ __forceinline__ uint32_t mx_get2_bf16(uint32_t word, float scale) {
  return __builtin_bit_cast(uint32_t, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, BYTE));
}

}  // namespace foremoe
