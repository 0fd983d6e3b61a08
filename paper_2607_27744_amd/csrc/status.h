// Status reporting and argument checks shared by the C ABI files.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/rocs.h"

namespace rocs {

// Sets the calling thread's message and returns the status.
int32_t fail(rocs_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the message and returns ROCS_OK.
int32_t ok();
int32_t launch_failed(const char* name, hipError_t e);

inline bool aligned(const void* p, uintptr_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}

// Byte ranges [a, a + an) and [b, b + bn) intersect.
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  if (a == nullptr || b == nullptr || an == 0 || bn == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + bn && y < x + an;
}

inline size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

inline bool valid_dtype(int32_t d) { return d == ROCS_DTYPE_F32 || d == ROCS_DTYPE_BF16; }
inline size_t esize(int32_t d) { return d == ROCS_DTYPE_BF16 ? 2 : 4; }

constexpr int64_t kMaxI32 = 2147483647;

}  // namespace rocs
