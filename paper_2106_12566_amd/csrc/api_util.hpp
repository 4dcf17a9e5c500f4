// Host-side helpers of the C ABI's entry points (api.hip, api_decay.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "krpe.h"

namespace krpe {

// Sets the calling thread's krpe_last_error() text and returns `s`.
krpe_status_t fail(krpe_status_t s, const std::string& msg);
void clear_error();

inline size_t align_up(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

struct Range {
  const void* p;
  size_t bytes;
};
inline bool overlaps(Range a, Range b) {
  if (a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

inline size_t dtype_size(int dt) { return dt == KRPE_BF16 ? 2 : 4; }

inline krpe_status_t hip_check(hipError_t e, const char* what) {
  if (e == hipSuccess) return KRPE_OK;
  return fail(KRPE_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace krpe
