// Rows of a 4-bit cache: blocks of 32 values along a head (fp4 e2m1 codes, two a byte, the even element in the low
// half) that share one power of two (e8m0, a byte).  A block of largest magnitude a is scaled by 2^e, e the smallest
// integer in [-127, 125] with a <= 7 * 2^e; a value becomes the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} to x / 2^e,
// ties to the even code.  7 is where 6 stops being the nearest value of a grid that went on, so the largest value of
// a block is off by half a step at most, like the others, and a power-of-two scale keeps every step exact: bf16 to
// code, and code to bf16.  Both directions are one gfx950 conversion instruction per two values.
#pragma once

#include "common.h"

namespace sonic {

constexpr int kQ4Block = 32;
constexpr uint32_t kQ4NanScale = 255;   // a block that held an infinity or a NaN: all of it is NaN

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Largest magnitude of the 2 N bf16 values in w, as a bf16 bit pattern (NaN patterns compare above infinity).
template <int N> __device__ __forceinline__ uint32_t q4_top(const uint32_t (&w)[N]) {
  u16x2 t = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  return max(static_cast<uint32_t>(t[0]), static_cast<uint32_t>(t[1]));
}

// The scale byte (e + 127) of a block of largest magnitude `top`: a = 2^(E - 127) (1 + m / 128) needs
// e = E - 129, or one more when 1 + m / 128 passes 1.75 (m > 96, which 31 carries into E).
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t top) {
  const int s = static_cast<int>((top + 31) >> 7) - 2;
  return top >= 0x7F80u ? kQ4NanScale : static_cast<uint32_t>(min(max(s, 0), 252));
}

// A scale byte as the operand of the conversions, which look at its exponent bits only.
__device__ __forceinline__ float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight bf16 values to eight codes.
__device__ __forceinline__ uint32_t q4_encode8(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t byte) {
  if (byte == kQ4NanScale) return 0;
  const float s = q4_scale(byte);
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, __builtin_bit_cast(bf16x2, w0), s, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, __builtin_bit_cast(bf16x2, w1), s, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, __builtin_bit_cast(bf16x2, w2), s, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, __builtin_bit_cast(bf16x2, w3), s, 3);
  return u;
}

// Eight codes to eight bf16 values, exactly.
__device__ __forceinline__ bf16x8 q4_decode8(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  const auto ab = __builtin_shufflevector(a, b, 0, 1, 2, 3), cd = __builtin_shufflevector(c, d, 0, 1, 2, 3);
  return __builtin_shufflevector(ab, cd, 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace sonic
