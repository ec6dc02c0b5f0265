// Host-side checks of the entry points over a bounded view of the prefix, built
// like abi_harness.cpp (sanitizers on the host code, stub launchers that launch
// nothing): the launch parameters describe the problem, the partials lie in the
// caller's workspace, and a workspace for the longest prefix serves shorter ones.
#include <cstdio>
#include <cstring>
#include <random>

#include "view.hpp"
#include "zarya.h"

static int g_fail = 0, g_checks = 0, g_launches = 0, g_few = 0, g_split = 0;
#define CHECK(c)                                                        \
  do {                                                                  \
    ++g_checks;                                                         \
    if (!(c)) {                                                         \
      std::printf("FAIL %s:%d: %s\n", __FILE__, __LINE__, #c);          \
      ++g_fail;                                                         \
    }                                                                   \
  } while (0)

static uintptr_t g_ws_lo = 0, g_ws_hi = 0;
static bool in_ws(const void* p, size_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return a >= g_ws_lo && a + bytes <= g_ws_hi;
}

namespace zarya {

static zarya_attn_window g_window;
static bool g_codes;

template <class P>
static void check_view(const P& p, bool codes) {
  ++g_launches;
  CHECK(codes == g_codes);
  CHECK(p.T == p.S * p.L && p.G * p.Hkv == p.Hq && p.rows_total == p.B * p.Hq * p.T);
  CHECK(p.window >= 1 && p.sinks >= 0);
  CHECK(g_window.window > 0 ? p.window == g_window.window && p.sinks == g_window.sinks
                            : p.window == 2147483647 && p.sinks == 0);
}

static hipError_t check_bf16(const ViewParams& all, int head_dim, bool codes) {
  check_view(all, codes);
  CHECK(all.n_split >= 1 && all.n_split <= 64 && all.R == all.G * all.T);
  CHECK((int64_t)all.n_rb * all.rows_per_block >= all.R && (int64_t)(all.n_rb - 1) * all.rows_per_block < all.R);
  CHECK(all.n_items == all.B * all.Hkv * all.n_split * all.n_rb);
  if (all.n_split > 1) {
    ++g_split;
    CHECK(in_ws(all.part_o, (size_t)all.n_split * all.rows_total * head_dim * 4));
    CHECK(in_ws(all.part_lse, (size_t)all.n_split * all.rows_total * 4));
    CHECK((uintptr_t)all.part_lse >= (uintptr_t)all.part_o + (size_t)all.n_split * all.rows_total * head_dim * 4);
  }
  int64_t next = 0;  // the grids cover the items once, in order
  for_each_view_launch(all, [&](const ViewParams& p) {
    CHECK(p.item0 == next && p.n_items >= 1 && p.n_items <= kAttnMaxGrid && p.per_xcd * 8 >= p.n_items);
    CHECK(!p.heavy_first || (p.n_split == 1 && p.per_xcd * 8 == p.n_items && p.per_xcd % p.n_rb == 0 && p.item0 == 0));
    next += p.n_items;
  });
  CHECK(next == all.n_items);
  return hipErrorNoDevice;
}

hipError_t launch_slot_view_bf16(const ViewParams& p, int d, bool codes, hipStream_t) {
  CHECK(p.rows_per_block == kAttnRowsPerBlock || p.rows_per_block == kAttnWideRowsPerBlock);
  return check_bf16(p, d, codes);
}
hipError_t launch_slot_view_few(const ViewParams& p, int d, bool codes, hipStream_t) {
  ++g_few;
  CHECK(p.rows_per_block == 16 || p.rows_per_block == 32);
  CHECK(!p.heavy_first);
  return check_bf16(p, d, codes);
}
hipError_t launch_slot_view_f32(const ViewParams32& p, int, bool codes, hipStream_t) {
  check_view(p, codes);
  return hipErrorNoDevice;
}
hipError_t launch_kv_quantize(const KvQ4Params& p, hipStream_t) {
  ++g_launches;
  CHECK(p.N >= 1 && p.N <= p.C && p.cache.k_codes && p.cache.v_scales);
  return hipErrorNoDevice;
}
hipError_t launch_kv_dequantize(const KvQ4Params& p, hipStream_t s) { return launch_kv_quantize(p, s); }
hipError_t launch_kv_append_q4(const AppendQ4Params& p, hipStream_t) {
  ++g_launches;
  CHECK(p.S * p.L <= kAppendMaxTokens && p.S <= 1024 && p.cache.k_codes && p.cache.v_scales);
  return hipErrorNoDevice;
}

// the launchers of the other entry points, which nothing here reaches
#define UNUSED(name, type) \
  hipError_t name(const type&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_slot_attn_bf16(const AttnParams&, int, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_slot_attn_f32(const AttnParams32&, int, hipStream_t) { return hipErrorNoDevice; }
UNUSED(launch_slot_conf_bf16, ConfParams)
UNUSED(launch_slot_conf_f32, ConfParams)
UNUSED(launch_slot_conf_merge, ConfMergeParams)
UNUSED(launch_select_slots, SelectParams)
UNUSED(launch_verify_accept, AcceptParams)
UNUSED(launch_kv_append, AppendParams)
UNUSED(launch_mdm_reveal, RevealParams)

}  // namespace zarya

static void* fake(uintptr_t a) { return reinterpret_cast<void*>(a); }
static uint8_t* const kP = static_cast<uint8_t*>(fake(0x200000000ull));

static zarya_status call(const zarya_slot_attn_desc& d, const zarya_attn_window* w, bool codes, size_t ws) {
  void* wsp = ws ? fake(g_ws_lo) : nullptr;
  return codes ? zarya_slot_attn_q4(&d, w, kP, kP, kP, kP, kP, kP, kP, nullptr, nullptr, kP, nullptr, wsp, ws, nullptr)
               : zarya_slot_attn_window(&d, w, kP, kP, kP, kP, kP, nullptr, nullptr, kP, nullptr, wsp, ws, nullptr);
}

static size_t size_of(const zarya_slot_attn_desc& d, const zarya_attn_window* w, bool codes) {
  size_t ws = ~(size_t)0;
  CHECK((codes ? zarya_slot_attn_q4_workspace_size(&d, w, &ws) : zarya_slot_attn_window_workspace_size(&d, w, &ws)) ==
        ZARYA_OK);
  return ws;
}

int main() {
  std::mt19937_64 rng(7);
  for (int it = 0; it < 1500; ++it) {
    zarya_slot_attn_desc d{};
    d.batch = 1 + (int)(rng() % (rng() % 2 ? 64 : 3));
    d.n_kv_heads = 1 + (int)(rng() % 8);
    d.n_q_heads = d.n_kv_heads * (1 + (int)(rng() % 7));
    d.head_dim = rng() % 2 ? 64 : 128;
    d.prefix_len = (rng() % 5 == 0) ? (int)(rng() % 3) : (int)(rng() % 40000);
    d.kv_capacity = d.prefix_len + (int)(rng() % 300);
    d.n_slots = rng() % 2 ? 1 : 1 + (int)(rng() % 64);
    d.slot_len = rng() % 2 ? 1 : 1 + (int)(rng() % 32);
    d.softmax_scale = 0.088f;
    d.pass = (int)(rng() % 2);
    d.cross_slot = (int)(rng() % 2);
    d.dtype = (rng() % 5 == 0) ? ZARYA_DTYPE_F32 : ZARYA_DTYPE_BF16;
    d.prefix_splits = (rng() % 3 == 0) ? (int)(rng() % 65) : 0;
    const bool codes = rng() % 2;
    zarya_attn_window w{(int)(rng() % 3 ? 1 + rng() % 5000 : 2147483647u), (int)(rng() % 3 ? rng() % 100 : 2147483647u)};
    if (codes && rng() % 3 == 0) w = zarya_attn_window{0, 0};
    const zarya_attn_window* wp = codes && w.window == 0 && rng() % 2 ? nullptr : &w;
    zarya::g_window = w;
    zarya::g_codes = codes;
    const size_t ws = size_of(d, wp, codes);
    g_ws_lo = 0x100000000ull;
    g_ws_hi = g_ws_lo + ws;
    const int before = g_launches;
    CHECK(call(d, wp, codes, ws) == ZARYA_ERR_HIP && g_launches == before + 1 && std::strlen(zarya_last_error()) > 0);
    if (ws > 0) CHECK(call(d, wp, codes, ws - 1) == ZARYA_ERR_WORKSPACE_TOO_SMALL && g_launches == before + 1);
    if (d.prefix_splits == 0) {  // every shorter prefix fits
      zarya_slot_attn_desc s = d;
      for (int i = 0; i < 20; ++i) {
        s.prefix_len = (int)(rng() % (d.prefix_len + 1));
        CHECK(size_of(s, wp, codes) <= ws);
      }
    }
  }
  // more workgroups than a grid holds: batch * heads of single rows
  zarya_slot_attn_desc big{};
  big.batch = 400000;
  big.n_kv_heads = 8;
  big.n_q_heads = 8;
  big.head_dim = 64;
  big.n_slots = big.slot_len = 1;
  big.softmax_scale = 1.f;
  big.dtype = ZARYA_DTYPE_BF16;
  zarya::g_window = zarya_attn_window{5, 0};
  zarya::g_codes = false;
  CHECK(call(big, &zarya::g_window, false, 0) == ZARYA_ERR_HIP);

  zarya_kv_q4_desc q{2, 8, 128, 4096, 77, ZARYA_DTYPE_BF16};
  int before = g_launches;
  CHECK(zarya_kv_quantize(&q, kP, kP, nullptr, nullptr, kP, kP, kP, kP, nullptr) == ZARYA_ERR_HIP);
  CHECK(zarya_kv_dequantize(&q, kP, kP, kP, kP, nullptr, kP, kP, nullptr) == ZARYA_ERR_HIP);
  zarya_kv_append_desc a{2, 8, 128, 4096, 64, 128, ZARYA_DTYPE_BF16};
  CHECK(zarya_kv_append_q4(&a, kP, kP, kP, (const int32_t*)kP, (int32_t*)kP, kP, kP, kP, kP, nullptr) == ZARYA_ERR_HIP);
  CHECK(g_launches == before + 3);
  q.n_rows = 0;  // nothing to do, nothing launched, no pointer looked at
  CHECK(zarya_kv_quantize(&q, nullptr, nullptr, nullptr, nullptr, kP, kP, kP, kP, nullptr) == ZARYA_OK);
  CHECK(g_launches == before + 3);
  CHECK(g_few > 100 && g_split > 100);
  std::printf("%d checks, %d failures, %d launches reached\n", g_checks, g_fail, g_launches);
  return g_fail == 0 ? 0 : 1;
}
