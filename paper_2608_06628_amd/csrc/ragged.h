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

// Sequences whose workgroups are taken by levels: sequence b has count(b) of them, at the levels
// count(b) - 1 .. 0, and the x-th of all comes after those of higher levels, so that where
// a workgroup's work grows with its level the longest go first, whatever the lengths.
// Items at levels above y are sum_b max(0, count(b) - 1 - y): the level is found by halving, in a
// lane's sequences' counts at a time, and the sequence among those that have the level.
constexpr int kLevelLanes = 4;  // sequences of a lane
constexpr int kMaxLevelled = kWave * kLevelLanes;

__device__ inline int ragged_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);  // row_ror:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false);
  auto f = [](int v) { return __builtin_bit_cast(float, v); };
  x += __builtin_bit_cast(int, xor16(f(x)));
  return __builtin_amdgcn_readfirstlane(x + __builtin_bit_cast(int, xor32(f(x))));
}

__device__ inline int ragged_most(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));
  auto f = [](int v) { return __builtin_bit_cast(float, v); };
  x = max(x, __builtin_bit_cast(int, xor16(f(x))));
  return __builtin_amdgcn_readfirstlane(max(x, __builtin_bit_cast(int, xor32(f(x)))));
}

// Finds the x-th workgroup's sequence and level (b = -1: there are fewer).
template <typename F>
__device__ inline int ragged_level(int n, int x, int lane, F count, int& level) {
  int c[kLevelLanes], most = 0;
#pragma unroll
  for (int i = 0; i < kLevelLanes; ++i) {
    c[i] = 0;
    if (i * kWave < n && lane + i * kWave < n) c[i] = count(lane + i * kWave);
    most = max(most, c[i]);
  }
  auto above = [&](int y) {  // workgroups at levels above y
    int t = 0;
#pragma unroll
    for (int i = 0; i < kLevelLanes; ++i) t += max(0, c[i] - 1 - y);
    return ragged_sum(t);
  };
  int lo = -1, hi = ragged_most(most) - 1;  // above(hi) <= x; above(lo) > x, or lo = -1
  if (above(-1) <= x) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (above(mid) <= x)
      hi = mid;
    else
      lo = mid;
  }
  level = hi;
  int rest = x - above(hi);
#pragma unroll
  for (int i = 0; i < kLevelLanes; ++i) {
    unsigned long long have = __ballot(c[i] > hi);
    const int k = __builtin_popcountll(have);
    if (rest < k) {
      for (int j = 0; j < rest; ++j) have &= have - 1;
      return i * kWave + __builtin_ctzll(have);
    }
    rest -= k;
  }
  return -1;
}

}  // namespace hyb
