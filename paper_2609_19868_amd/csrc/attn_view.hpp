// Bounded views of the prefix cache: a sliding window with sinks, and 4-bit codes.
//
// Places are counted in the committed order: prefix row j has place j, draft
// token t of a row with Pb prefix rows has place Pb + t.  A key at place j that
// the pass shows to a token at place i is visible when j < sinks or j > i - window.
//
// A block of 4-bit codes is 32 neighbouring elements of a row, in e2m1 (sign,
// magnitude 0, 1/2, 1, 3/2, 2, 3, 4 or 6), with one scale byte, the exponent field
// of a float32 power of two (255: not a number).  Conversions from it are exact
// in bf16: three significant bits times a power of two.
#pragma once

#include "common.hpp"

namespace zarya {

// The tiles of KT keys that hold what the tokens t0..t1 of a row block see: the
// prefix's sinks and window, then the draft tokens' (whose first keys are sinks
// where the prefix is shorter than the sinks).  Tile i of the list is keys
// [key0(i), key0(i) + KT) of the prefix (i < n_pre) or of the draft tokens; no
// tile is listed twice.
template <int KT>
struct KeyTiles {
  int n_ps, pw, n_pre, ds, n_ds, dw, nt;

  // lo, hi: the draft keys that the pass shows to any of the tokens
  __device__ __forceinline__ void list(int Pb, int t0, int lo, int hi, int window, int sinks) {
    const int edge = Pb + t0 - window + 1;  // first place inside the first token's window
    n_ps = (min(sinks, Pb) + KT - 1) / KT;
    const int w0 = max(min(max(edge, 0), Pb) / KT, n_ps);
    pw = w0 - n_ps;
    n_pre = n_ps + max(0, (Pb + KT - 1) / KT - w0);
    const int sd = min(sinks - Pb, hi);  // draft keys below this are sinks
    ds = lo / KT;
    n_ds = sd > lo ? (sd + KT - 1) / KT - ds : 0;
    dw = max(max(lo, edge - Pb) / KT, ds + n_ds);
    nt = n_pre + n_ds + max(0, (hi + KT - 1) / KT - dw);
  }
  __device__ __forceinline__ int key0(int i) const {
    int k = i;
    if (i >= n_ps) k = i + pw;
    if (i >= n_pre) k = i - n_pre + ds;
    if (i >= n_pre + n_ds) k = i - n_pre - n_ds + dw;
    return k * KT;
  }
};

// Scale byte in the low bits of `b` -> the power of two that the conversions take
// (they look at the exponent field alone).
__device__ __forceinline__ float q4_scale(uint32_t b) { return __uint_as_float(b << 23); }

// Eight codes of one block (element 2 * i in the low half of byte i) -> bf16.
__device__ __forceinline__ bf16x8 q4_bf16x8(uint32_t codes, float scale) {
  bf16x2_t v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return __builtin_bit_cast(bf16x8, v);
}

// Four codes in the low 16 bits -> float32.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f32x4 q4_f32x4(uint32_t codes, float scale) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  return f32x4{a.x, a.y, b.x, b.y};
}

}  // namespace zarya
