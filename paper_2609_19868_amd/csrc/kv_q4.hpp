// Rows of keys and values into 4-bit blocks: the part that quantizing a prefix and
// appending accepted tokens share.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace zarya {

// Eight neighbouring elements as float32 (exact).
__device__ __forceinline__ void load_f32x8(const void* base, size_t element, int bf16, float x[8]) {
  if (bf16) {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + element);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
    const float* src = static_cast<const float*>(base) + element;
    const f32x4 a = load_f32x4(src), b = load_f32x4(src + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = a[e];
      x[4 + e] = b[e];
    }
  }
}

// One block of 32 elements by four neighbouring lanes (of a multiple of four), eight
// elements each: the lane's four bytes of codes, and the block's scale byte.
//
// The scale is the smallest power of two for which the largest magnitude a rounds
// to at most 6: floor(log2 a) - 2, and one more from a mantissa of 1.75 on (7 is
// halfway between 6 and 8 and rounds to 8, whose code is even), so that no element
// is off by more than half a step.  The byte is held to 252, of which 6 is still
// finite in bf16 and float32: only there, from 7 * 2^125 on, are values cut to 6.
// A block with a NaN or an infinity gets the byte 255, which reads as NaN.
__device__ __forceinline__ uint32_t q4_codes(const float x[8], uint32_t& byte) {
  uint32_t top = 0;  // magnitudes compare as integers, infinities and NaN above all
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));  // lane ^ 1
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));  // lane ^ 2
  const int exponent = (int)(top >> 23) - 2 + ((top & 0x7fffffu) >= 0x600000u ? 1 : 0);
  byte = top >= 0x7f800000u ? 255u : (uint32_t)min(max(exponent, 0), 252);
  const float scale = __uint_as_float(byte << 23);
  uint32_t codes = 0;  // nearest magnitude, halves to the even code
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  return byte == 255u ? 0u : codes;
}

// Piece `c` (eight elements) of a row of the cache, written by its lane.
__device__ __forceinline__ void store_q4(uint8_t* codes, uint8_t* scales, size_t row, int D, int c, const float x[8]) {
  uint32_t byte;
  const uint32_t w = q4_codes(x, byte);
  *reinterpret_cast<uint32_t*>(codes + row * (D / 2) + 4 * c) = w;
  if ((c & 3) == 0) scales[row * (D / 32) + c / 4] = (uint8_t)byte;
}

}  // namespace zarya
