// Device-side part shared by the kernels of the adapter linear (adapter.hip, linear.hip).
#pragma once

#include "common.h"
#include "layer.h"

namespace rocs {

// Adapter of row n as the first launch has written it. A row that belongs to no request
// (offsets that do not start at 0) has what the workspace held: anything outside the adapters
// is none.
__device__ __forceinline__ int adapter_at(const LowRank& lr, int64_t n) {
  const int id = lr.aid[n];
  return (uint32_t)id < (uint32_t)lr.adapters ? id : -1;
}

}  // namespace rocs
