// packed_rows.h -- which sequence a packed row, or a tile of them, belongs to (device side).
#pragma once

#include <stdint.h>

namespace bana {

// row_begin[b], whatever it holds, as a row number or the end of the rows.
__device__ __forceinline__ int row_start(const int32_t* __restrict__ row_begin, int b, int rows) {
  return min(max(row_begin[b], 0), rows);
}

// The last b in [0, B) with first(b) <= x, first not decreasing (0 if there is none): all lanes of the
// wavefront look at 64 places of the remaining range at once, so 4096 sequences take two rounds of loads.
template <typename F>
__device__ __forceinline__ int last_at_most(int B, int x, int lane, F first) {
  int lo = 0, n = B;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int at = lo + lane * step;
    const bool ok = lane * step < n && first(at) <= x;
    const int below = max((int)__popcll(__ballot(ok)) - 1, 0);  // none: the first
    lo += below * step;
    n = min(step, n - below * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace bana
