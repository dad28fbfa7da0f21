// The 4-bit cache: E2M1 codes with one E8M0 scale per token, KV head and 32 channels (the OCP microscaling format MXFP4), which
// the gfx950 conversion instructions read and write two at a time.
//
//   k_codes [pages, Hkv, g, d/2]           byte i of a token: channels 2 i (low four bits) and 2 i + 1
//   v_codes [pages, Hkv, g/4, 16, d/32, 4] byte [q][r][j][t]: channels 32 j + r (low four bits) and 32 j + 16 + r of token 4 q + t
//   scales  [pages, Hkv, 2, g, d/32]       keys' scale bytes, then values'; byte b stands for 2^(b - 127), 255 for NaN
//
// A byte holds codes of one token only, so that a token is appended without reading what lies beside it.  The orders are those in which
// the matrix cores take their operands: sixteen tokens' keys are 16 bytes per lane (a token's 32 channels under one scale), sixteen
// tokens' values are 16 bytes per lane as well (four tokens, all channels that are r modulo 16), each read in one go and in lane order.
#pragma once
#include "losa_device.h"
#include "losa_internal.h"

namespace losa {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;

// Limits of a group's scale byte.  Keys: every number is a normal bfloat16.  Values: every number is exact in half precision
// (2^-23 .. 49152), in which the attention multiplies them with the probabilities.
constexpr int kKeyScaleMin = 2, kKeyScaleMax = 252, kValueScaleMin = 105, kValueScaleMax = 140, kScaleNaN = 255;

// Scale byte of a group whose largest magnitude is `top`: the power of two X with 3.5 X <= top < 7 X, so that the largest number
// rounds to 6 X at most.  (In the bits of a float: a quarter added to the mantissa carries into the exponent from 1.75 on.)
__device__ __forceinline__ int scale_byte(float top, int least, int most) {
  const int e = (int)((__float_as_uint(top) + 0x200000u) >> 23) - 2;
  return top < INFINITY ? min(max(e, least), most) : kScaleNaN;   // (NaN compares false)
}
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two numbers' codes in byte SEL of a dword, `a` in its low four bits; to nearest, ties to even, saturating at 6.
template <int SEL>
__device__ __forceinline__ uint32_t put_codes(uint32_t old, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, SEL);
}
// ... and back.
template <int SEL>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
template <int SEL>
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
}

}  // namespace losa
