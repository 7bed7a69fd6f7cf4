// The steps of the wavefront's search in ascending entries, apart from the wavefront's instructions so that they compile for the host too.
#pragma once

namespace ekv {

// The last of n entries that is not above a value.  at_most(lo, n, step): how many of the entries lo + lane * step, lane * step < n, of a
// wavefront's 64 lanes are not above it.  0 <= result < n whatever at_most counts: where the first entry is above the value, or
// entries do not ascend, the result is an entry all the same, and whoever has to know whether it is above the value compares it.
template <typename F> __device__ __forceinline__ int last_at_most_by_64(int n, F&& at_most) {
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) >> 6, counted = at_most(lo, n, step), k = counted > 0 ? counted - 1 : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return lo;
}

}  // namespace ekv
