// ragged.h -- sequences of different lengths one after the other in one array, whose
// starts are on the device.
#pragma once

#include "device.h"

namespace hyb {

// First row of sequence b: starts [.. B] are not falling; clamped to 0 .. n, and 0 for the
// first, so that whatever they hold no row outside the array is touched.
__device__ inline int ragged_start(const int32_t* starts, int b, int n) { return b == 0 ? 0 : min(max(starts[b], 0), n); }

// The last of n sequences whose first place is at most x; place(0) <= x, and place does
// not fall.  The whole wave, by one look at 64 sequences (two for 4096).
template <typename F>
__device__ inline int ragged_find(int n, long x, int lane, F place) {
  int lo = 0, hi = n;  // it is among lo .. hi - 1
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, b = lo + lane * step;
    const bool by = b < hi && place(b) <= x;
    lo += step * max(0, __builtin_popcountll(__ballot(by)) - 1);
    hi = min(hi, lo + step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace hyb
