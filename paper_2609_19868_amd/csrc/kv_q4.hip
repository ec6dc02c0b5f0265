// A prefix into the 4-bit cache and out of it (gfx950).
//
// Both directions only move bytes: 2 D elements in and 2 (D/2 + D/32) bytes out per
// row and head, or the other way round, bound by HBM.  A lane takes 16 bytes of
// elements (32 of float32 when quantizing: a block is four lanes), so that a wave
// reads and writes whole lines; a workgroup of 256 takes neighbouring rows of one
// head, K and V, with every load of a lane requested before the first is used.  The
// elements are read and written past the caches' order (non-temporal): 8 x 8 x 16384
// rows of bf16, D = 128, 680 MB: in 118 us, out 109, 5.7 and 6.2 TB/s (a copy reaches
// 5.2); without 127 and 120.
#include <algorithm>

#include "attn_view.hpp"
#include "common.hpp"
#include "kv_q4.hpp"
#include "view.hpp"

namespace zarya {

namespace {

constexpr int kThreads = 256;
// pieces of K and of V per lane (in: 2 and 8 no faster; out: 4 126 us)
constexpr int kPiecesIn = 4, kPiecesOut = 2;

// Chunks of rows of every head, for lanes of E elements and `pieces` rows each:
// f(first row of the head in [B, Hkv, N], first row in the cache, this lane's first
// row, its place in the row, rows asked for)
template <int D, int E, int PIECES, class F>
__device__ __forceinline__ void each_chunk(const KvQ4Params& p, F&& f) {
  constexpr int RPC = kThreads * PIECES / (D / E);
  const int per_head = (p.N + RPC - 1) / RPC;
  const int64_t n = (int64_t)p.B * p.Hkv * per_head;
  for (int64_t w = blockIdx.x; w < n; w += gridDim.x) {
    const int bg = (int)(w / per_head), chunk = (int)(w % per_head), b = bg / p.Hkv;
    const int len = p.lens ? min(max(p.lens[b], 0), p.N) : p.N;
    const int start = p.starts ? p.starts[b] : 0;
    if (start < 0 || (int64_t)start + len > p.C) continue;  // a row that does not fit stays as it is
    const int r0 = chunk * RPC + threadIdx.x / (D / E), c = threadIdx.x % (D / E);
    f((size_t)bg * p.N, (size_t)bg * p.C + start, r0, c, len);
  }
}

}  // namespace

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv_quantize_kernel(KvQ4Params p) {
  constexpr int STEP = kThreads / (D / 8);  // rows between a lane's pieces
  each_chunk<D, 8, kPiecesIn>(p, [&](size_t src, size_t dst, int r0, int c, int len) {
    Elements8<BF16> k[kPiecesIn], v[kPiecesIn];
#pragma unroll
    for (int i = 0; i < kPiecesIn; ++i) {
      const size_t at = (src + min(r0 + i * STEP, max(len - 1, 0))) * D + 8 * c;
      k[i] = load_elements8<BF16, true>(p.k, at);
      v[i] = load_elements8<BF16, true>(p.v, at);
    }
#pragma unroll
    for (int i = 0; i < kPiecesIn; ++i) {
      const int r = r0 + i * STEP;
      if (r < len) {  // the same for the four lanes of a block
        store_q4<BF16>(p.cache.k_codes, p.cache.k_scales, dst + r, D, c, k[i]);
        store_q4<BF16>(p.cache.v_codes, p.cache.v_scales, dst + r, D, c, v[i]);
      }
    }
  });
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv_dequantize_kernel(KvQ4Params p) {
  constexpr int E = BF16 ? 8 : 4;  // elements of 16 bytes
  constexpr int STEP = kThreads / (D / E);
  each_chunk<D, E, kPiecesOut>(p, [&](size_t dst, size_t src, int r0, int c, int len) {
    uint32_t code[2][kPiecesOut], byte[2][kPiecesOut];
#pragma unroll
    for (int i = 0; i < kPiecesOut; ++i) {
      const size_t row = src + min(r0 + i * STEP, max(len - 1, 0));
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint8_t* codes = (w ? p.cache.v_codes : p.cache.k_codes) + row * (D / 2) + c * (E / 2);
        if constexpr (BF16) {
          code[w][i] = *reinterpret_cast<const uint32_t*>(codes);
        } else {
          code[w][i] = *reinterpret_cast<const uint16_t*>(codes);
        }
        byte[w][i] = (w ? p.cache.v_scales : p.cache.k_scales)[row * (D / 32) + c * E / 32];
      }
    }
#pragma unroll
    for (int i = 0; i < kPiecesOut; ++i) {
      const int r = r0 + i * STEP;
      if (r >= len) continue;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const float scale = q4_scale(byte[w][i]);
        const size_t at = (dst + r) * D + E * c;
        if constexpr (BF16) {
          __builtin_nontemporal_store(q4_bf16x8(code[w][i], scale),
                                      reinterpret_cast<bf16x8*>(static_cast<uint16_t*>(w ? p.v : p.k) + at));
        } else {
          __builtin_nontemporal_store(q4_f32x4(code[w][i], scale),
                                      reinterpret_cast<f32x4*>(static_cast<float*>(w ? p.v : p.k) + at));
        }
      }
    }
  });
}

namespace {

template <class Kernel>
void launch_chunks(Kernel kernel, int rows, const KvQ4Params& p, hipStream_t stream) {
  const int64_t chunks = (int64_t)p.B * p.Hkv * ((p.N + rows - 1) / rows);
  kernel<<<dim3((int)std::min<int64_t>(chunks, kAttnMaxGrid)), dim3(kThreads), 0, stream>>>(p);
}

template <int D, bool BF16>
void launch_quantize_as(const KvQ4Params& p, hipStream_t stream) {
  launch_chunks(kv_quantize_kernel<D, BF16>, kThreads * kPiecesIn / (D / 8), p, stream);
}

template <int D, bool BF16>
void launch_dequantize_as(const KvQ4Params& p, hipStream_t stream) {
  launch_chunks(kv_dequantize_kernel<D, BF16>, kThreads * kPiecesOut / (D / (BF16 ? 8 : 4)), p, stream);
}

}  // namespace

hipError_t launch_kv_quantize(const KvQ4Params& p, hipStream_t stream) {
  if (p.D == 128) {
    p.bf16 ? launch_quantize_as<128, true>(p, stream) : launch_quantize_as<128, false>(p, stream);
  } else {
    p.bf16 ? launch_quantize_as<64, true>(p, stream) : launch_quantize_as<64, false>(p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_kv_dequantize(const KvQ4Params& p, hipStream_t stream) {
  if (p.D == 128) {
    p.bf16 ? launch_dequantize_as<128, true>(p, stream) : launch_dequantize_as<128, false>(p, stream);
  } else {
    p.bf16 ? launch_dequantize_as<64, true>(p, stream) : launch_dequantize_as<64, false>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace zarya
