// A prefix into the 4-bit cache and out of it (gfx950).
//
// Both directions only move bytes: 2 D elements in and 2 (D/2 + D/32) bytes out per
// row and head, or the other way round, bound by HBM.  A lane takes eight elements
// (16 bytes in bf16, 4 bytes of codes), so that a wave reads and writes whole
// lines; a workgroup of 256 takes 64 neighbouring rows (D = 128) of one head, K and
// V, with every load of a lane requested before the first is used.
#include <algorithm>

#include "attn_view.hpp"
#include "common.hpp"
#include "kernels.hpp"
#include "kv_q4.hpp"

namespace zarya {

namespace {

constexpr int kThreads = 256;
constexpr int kPieces = 4;  // of K and of V, per lane

template <int D>
constexpr int rows_per_chunk() {
  return kThreads * kPieces / (D / 8);
}

// f(first row of the head in [B, Hkv, N], first row in the cache, this lane's first
// row and its piece, rows asked for) for every chunk of rows of every head
template <int D, class F>
__device__ __forceinline__ void each_chunk(const KvQ4Params& p, F&& f) {
  constexpr int RPC = rows_per_chunk<D>();
  const int per_head = (p.N + RPC - 1) / RPC;
  const int64_t n = (int64_t)p.B * p.Hkv * per_head;
  for (int64_t w = blockIdx.x; w < n; w += gridDim.x) {
    const int bg = (int)(w / per_head), chunk = (int)(w % per_head), b = bg / p.Hkv;
    const int len = p.lens ? min(max(p.lens[b], 0), p.N) : p.N;
    const int start = p.starts ? p.starts[b] : 0;
    if (start < 0 || (int64_t)start + len > p.C) continue;  // a row that does not fit stays as it is
    const int r0 = chunk * RPC + threadIdx.x / (D / 8), c = threadIdx.x % (D / 8);
    f((size_t)bg * p.N, (size_t)bg * p.C + start, r0, c, len);
  }
}

}  // namespace

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv_quantize_kernel(KvQ4Params p) {
  constexpr int STEP = kThreads / (D / 8);  // rows between a lane's pieces
  each_chunk<D>(p, [&](size_t src, size_t dst, int r0, int c, int len) {
    float k[kPieces][8], v[kPieces][8];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const size_t at = (src + min(r0 + i * STEP, max(len - 1, 0))) * D + 8 * c;
      load_f32x8(p.k, at, BF16, k[i]);
      load_f32x8(p.v, at, BF16, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = r0 + i * STEP;
      if (r < len) {  // the same for the four lanes of a block
        store_q4(p.cache.k_codes, p.cache.k_scales, dst + r, D, c, k[i]);
        store_q4(p.cache.v_codes, p.cache.v_scales, dst + r, D, c, v[i]);
      }
    }
  });
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv_dequantize_kernel(KvQ4Params p) {
  constexpr int STEP = kThreads / (D / 8);
  each_chunk<D>(p, [&](size_t dst, size_t src, int r0, int c, int len) {
    uint32_t code[2][kPieces], byte[2][kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const size_t row = src + min(r0 + i * STEP, max(len - 1, 0));
      code[0][i] = *reinterpret_cast<const uint32_t*>(p.cache.k_codes + row * (D / 2) + 4 * c);
      code[1][i] = *reinterpret_cast<const uint32_t*>(p.cache.v_codes + row * (D / 2) + 4 * c);
      byte[0][i] = p.cache.k_scales[row * (D / 32) + c / 4];
      byte[1][i] = p.cache.v_scales[row * (D / 32) + c / 4];
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = r0 + i * STEP;
      if (r >= len) continue;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const float scale = q4_scale(byte[w][i]);
        const size_t at = (dst + r) * D + 8 * c;
        if constexpr (BF16) {
          *reinterpret_cast<bf16x8*>(static_cast<uint16_t*>(w ? p.v : p.k) + at) = q4_bf16x8(code[w][i], scale);
        } else {
          float* out = static_cast<float*>(w ? p.v : p.k) + at;
          store_f32x4(out, q4_f32x4(code[w][i], scale));
          store_f32x4(out + 4, q4_f32x4(code[w][i] >> 16, scale));
        }
      }
    }
  });
}

namespace {

template <class Kernel>
void launch_chunks(Kernel kernel, int rpc, const KvQ4Params& p, hipStream_t stream) {
  const int64_t chunks = (int64_t)p.B * p.Hkv * ((p.N + rpc - 1) / rpc);
  kernel<<<dim3((int)std::min<int64_t>(chunks, kAttnMaxGrid)), dim3(kThreads), 0, stream>>>(p);
}

}  // namespace

hipError_t launch_kv_quantize(const KvQ4Params& p, hipStream_t stream) {
  if (p.D == 128) {
    launch_chunks(p.bf16 ? kv_quantize_kernel<128, true> : kv_quantize_kernel<128, false>, rows_per_chunk<128>(), p, stream);
  } else {
    launch_chunks(p.bf16 ? kv_quantize_kernel<64, true> : kv_quantize_kernel<64, false>, rows_per_chunk<64>(), p, stream);
  }
  return hipGetLastError();
}

hipError_t launch_kv_dequantize(const KvQ4Params& p, hipStream_t stream) {
  if (p.D == 128) {
    launch_chunks(p.bf16 ? kv_dequantize_kernel<128, true> : kv_dequantize_kernel<128, false>, rows_per_chunk<128>(), p,
                  stream);
  } else {
    launch_chunks(p.bf16 ? kv_dequantize_kernel<64, true> : kv_dequantize_kernel<64, false>, rows_per_chunk<64>(), p,
                  stream);
  }
  return hipGetLastError();
}

}  // namespace zarya
