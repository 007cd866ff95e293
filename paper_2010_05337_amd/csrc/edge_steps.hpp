// The edges [beg, end) of a row in steps of U: step(e, k, at) for e = 0, U, ..
// below the row's count k, with at(u) the edge of slot u (the step's first one
// for a slot past the row's end, u >= k - e).  A row may have up to 2^31 - 1
// edges: no sum goes past its count, so none past an int32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gmb {

template <int U, typename Step>
__device__ __forceinline__ void edge_steps(int32_t beg, int32_t end, Step&& step) {
  const int32_t k = end - beg;
  if (k <= 0) return;
  for (int32_t e = 0;; e += U) {
    step(e, k, [=](int u) { return beg + (u < k - e ? e + u : e); });
    if (k - e <= U) break;
  }
}

}  // namespace gmb
