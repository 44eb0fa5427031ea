// packed_rows.h -- which sequence a packed row, or a tile of them, belongs to (device side).
#pragma once

#include <stdint.h>

namespace bana {

// row_begin[b], whatever it holds, as a row number or the end of the rows.
__device__ __forceinline__ int row_start(const int32_t* __restrict__ row_begin, int b, int rows) {
  return min(max(row_begin[b], 0), rows);
}

// A sequence, its rows and its entry of an array [B].
struct SeqRows {
  int b, begin, end, value;
};

// The last b in [0, B) with first(b, row_begin[b]) <= x, first increasing (0 if there is none), for every lane of the
// wavefront.  One load looks at 64 neighbours of where it would be if all sequences had as many rows (x * per_x), and
// at their values, and mostly settles it; otherwise each round looks at 64 places of the remaining range, so 4096
// sequences take two more.  (2048 single tokens, window 64: 203 us, by rounds alone 217.)
template <typename F>
__device__ __forceinline__ SeqRows find_rows(const int32_t* __restrict__ row_begin, const int32_t* __restrict__ values,
                                             int rows, int B, int x, float per_x, int lane, F first) {
  if (B > 1) {
    const int near = min(max((int)((float)x * per_x) - 31, 0), max(B - 63, 0)), at = near + lane;
    const int start = row_start(row_begin, min(at, B), rows), value = values[min(at, B - 1)];
    const int n_ok = (int)__popcll(__ballot(at < B && first(at, start) <= x));
    if (n_ok < 64 && (n_ok > 0 || near == 0)) {
      const int i = max(n_ok - 1, 0);
      return {near + i, __builtin_amdgcn_readlane(start, i), __builtin_amdgcn_readlane(start, i + 1),
              __builtin_amdgcn_readlane(value, i)};
    }
  }
  int lo = 0, n = B;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int b = lo + lane * step;
    const bool ok = lane * step < n && first(b, row_start(row_begin, b, rows)) <= x;
    const int below = max((int)__popcll(__ballot(ok)) - 1, 0);  // none: the first
    lo += below * step;
    n = min(step, n - below * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return {lo, row_start(row_begin, lo, rows), row_start(row_begin, lo + 1, rows), values[lo]};
}

}  // namespace bana
