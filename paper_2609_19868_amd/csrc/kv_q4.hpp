// Rows of keys and values into 4-bit blocks: the part that quantizing a prefix and
// appending accepted tokens share.
#pragma once

#include "common.hpp"
#include "view.hpp"

namespace zarya {

// Eight neighbouring elements as they are stored.  ONCE: in bf16 past the caches'
// order (a float32 lane's two pieces are halves of the same lines and need them).
template <bool BF16>
struct Elements8;
template <>
struct Elements8<true> {
  uint32_t w[4];
};
template <>
struct Elements8<false> {
  f32x4 a, b;
};
template <bool BF16, bool ONCE>
__device__ __forceinline__ Elements8<BF16> load_elements8(const void* base, size_t element) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (BF16) {
    const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + element);
    const u32x4 v = ONCE ? __builtin_nontemporal_load(src) : *src;
    return {{v[0], v[1], v[2], v[3]}};
  } else {
    const float* src = static_cast<const float*>(base) + element;
    return {load_f32x4(src), load_f32x4(src + 4)};
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
//
// Magnitudes compare as integers, infinities and NaN above all others; in bf16 two of
// them a word.
template <bool BF16>
__device__ __forceinline__ uint32_t q4_codes(const Elements8<BF16>& x, uint32_t& byte) {
  constexpr int MANT = BF16 ? 7 : 23;  // bits of the mantissa
  uint32_t top;
  if constexpr (BF16) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = __builtin_bit_cast(u16x2, x.w[e] & 0x7fff7fffu);
    const u16x2 t = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
    top = max((uint32_t)t[0], (uint32_t)t[1]);
  } else {
    top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      top = max(top, max(__float_as_uint(x.a[e]) & 0x7fffffffu, __float_as_uint(x.b[e]) & 0x7fffffffu));
  }
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));  // lane ^ 1
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));  // lane ^ 2
  const int exponent = (int)(top >> MANT) - 2 + ((top & ((1u << MANT) - 1)) >= (3u << (MANT - 2)) ? 1 : 0);
  byte = top >= 255u << MANT ? 255u : (uint32_t)min(max(exponent, 0), 252);
  const float scale = __uint_as_float(byte << 23);
  uint32_t codes = 0;  // nearest magnitude, halves to the even code
  if constexpr (BF16) {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x.w[0]), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x.w[1]), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x.w[2]), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, x.w[3]), scale, 3);
  } else {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.a[0], x.a[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.a[2], x.a[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.b[0], x.b[1], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.b[2], x.b[3], scale, 3);
  }
  return byte == 255u ? 0u : codes;
}

// Piece `c` (eight elements) of a row of the cache, written by its lane.
template <bool BF16>
__device__ __forceinline__ void store_q4(uint8_t* codes, uint8_t* scales, size_t row, int D, int c,
                                         const Elements8<BF16>& x) {
  uint32_t byte;
  const uint32_t w = q4_codes<BF16>(x, byte);
  *reinterpret_cast<uint32_t*>(codes + row * (D / 2) + 4 * c) = w;
  if ((c & 3) == 0) scales[row * (D / 32) + c / 4] = (uint8_t)byte;
}

}  // namespace zarya
