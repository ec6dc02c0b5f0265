// Host helpers shared by the C ABI's sources (api.hip, api_view.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "zarya.h"

namespace zarya {

constexpr int64_t kI32Max = 2147483647;

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Stores the message of zarya_last_error and returns `st`.
zarya_status fail(zarya_status st, const char* fmt, ...);
zarya_status hip_status(hipError_t e, const char* what);

zarya_status check_attn_desc(const zarya_slot_attn_desc* d);
zarya_status check_append_desc(const zarya_kv_append_desc* d);

}  // namespace zarya
