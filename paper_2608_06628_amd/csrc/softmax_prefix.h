// softmax_prefix.h -- what the kernels that attend over a cached prefix share:
// which of a request's keys its queries see, how the requests' keys are cut into
// ranges, the merge of the ranges' partial results, and their launch.
#pragma once

#include <algorithm>

#include "device.h"
#include "launch.h"

namespace hyb {

// WIN below: 0 the whole prefix, 1 its last `window` tokens and first n_sinks, 2 the
// same where the cache's tiles hold cached tokens only (an 8-bit cache, whose last tile
// is filled up, hidden, so that the block has a tile of its own).

// Keys of one split range at most: 32768 cached keys and a block fit one, and
// the page numbers of so many leave room for four of the paged ring's
// workgroups on a CU at d = 64 (65536 would leave room for three).
constexpr int kMaxRange = 49152;
// pages of one range at the smallest page size (32), unaligned ends included
constexpr int kMaxRangePages = kMaxRange / 32 + 2;

// Page of cached token j of a request (page table row ptab), clamped to the
// pool.
__device__ inline int sp_page(const SoftmaxPrefixArgs& a, const int32_t* ptab, int j) {
  const int pg = ptab[j >> a.page_shift];
  return min(max(pg, 0), a.n_pages - 1);
}

// Active tokens of request b's block.
template <int WIN>
__device__ inline int sp_block(const SoftmaxPrefixArgs& a, int b) {
  if constexpr (WIN) {
    if (a.block_len) return min(max(a.block_len[b], 0), a.s.L);
  }
  return a.s.L;
}

// Keys of request b: its cached prefix (clamped) and the block.
template <int WIN>
__device__ inline int sp_keys(const SoftmaxPrefixArgs& a, int b) {
  const int P = min(max(a.prefix_len[b], 0), a.max_prefix);
  return (WIN == 2 ? (P + kTile - 1) / kTile * kTile : P) + sp_block<WIN>(a, b);
}

// With WIN a cached token is visible among the first n_sinks or the last
// `window` of the prefix: the keys hs .. he - 1 are hidden.  The tiles keep
// their places in the cache (so a tile still lies in one page), and those that
// are hidden whole are skipped: tile tv of the request's list is tile tv of
// its keys, or tv + skip from st on.  Of the list at most two tiles are hidden
// in part (the last of the sinks, the first of the window, or one that is
// both); their hidden rows read a visible row of the tile and are masked in
// the scores, so nothing of what they hold plays a part.
struct SpSeen {
  int hs = 0, he = 0;    // hidden keys (none: hs = he)
  int st = 0, skip = 0;  // tiles before the skipped ones; skipped tiles
  __device__ inline int tile(int tv) const { return tv < st ? tv : tv + skip; }
  __device__ inline bool hides(int j) const { return j >= hs && j < he; }
  // a tile's first key j0: whether some of the tile's keys are hidden, and the
  // row that stands in for them
  __device__ inline bool cuts(int j0) const { return j0 < he && j0 + kTile > hs && hs < he; }
  __device__ inline int stand_in(int j0) const { return he < j0 + kTile ? he : hs - 1; }
};
template <int WIN>
__device__ inline SpSeen sp_seen(const SoftmaxPrefixArgs& a, int b) {
  SpSeen v;
  if constexpr (WIN) {
    const int P = min(max(a.prefix_len[b], 0), a.max_prefix);
    const int w0 = P - min(a.window, P);
    if (a.n_sinks < w0) {
      v.hs = a.n_sinks;
      v.he = w0;
      v.st = (v.hs + kTile - 1) / kTile;
      // (8-bit: a window of nothing leaves nothing in the cache's last tile)
      v.skip = max(0, (WIN == 2 && w0 == P ? (P + kTile - 1) / kTile : w0 / kTile) - v.st);
    }
  }
  return v;
}

template <int WIN>
__device__ inline int sp_tiles(const SoftmaxPrefixArgs& a, int b) {
  if constexpr (WIN) {
    if (sp_block<WIN>(a, b) == 0) return 0;  // (nothing to answer)
  }
  return (sp_keys<WIN>(a, b) + kTile - 1) / kTile - sp_seen<WIN>(a, b).skip;
}

// How the requests' keys are cut.  The lengths are known on the device only,
// so every workgroup works the cut out for itself, from prefix_len alone and
// with the same result: request b gets ceil(tiles_b / c) ranges, numbered
// through over the requests (so that the workgroups that have a range come first
// and spread over the chip; a fixed number of places per request took 8 paged
// requests of 1 to 4096 keys from 29 to 34 us), and range s of request b takes
// an even share of its tiles.  The tiles per range c is the
// candidate with the least estimated time (in whole numbers, so that every kernel
// finds the same).  Per KV head, `sat` workgroups use the memory fully and the
// chip holds `slots` of them at once.  Up to `sat` ranges take the time of the
// longest.  More, as far as they all fit, share the memory: the time of all their
// tiles (a tenth more, as they don't end together), or of the longest among as
// many neighbours as its CU has, half of whom end early, if that is more.  Ranges
// beyond that also pay for the part of the last round that stays empty.  A range
// costs its start, its partial result and that result's merge besides its tiles
// (sp_range_cost).  Candidates lie around the even share of `sat`; the
// last one cuts the longest request into limit / B ranges, so that all ranges fit
// the grid and the workspace.
// Equal cuts of max_prefix into n_split ranges, as it was, make 2048
// workgroups whatever the lengths: four rounds and a merge where one round of
// whole requests fills the chip (128 requests of 32768 keys: 1.70 against
// 1.54 ms, the loop below included), and ranges past a short request's end
// that still write, and have merged, an empty result (24 requests of 1 to
// 8192 keys: 104 against 76 us; 8 of 32768: 232 against 137 us).
struct SpCut {
  int slots, sat, limit;
  int layer;  // ranges per KV head that give every CU one workgroup
  int c;      // tiles per range where the host cuts, else 0
};
struct SpPlan {
  int c;       // tiles per range, before the even share
  bool whole;  // every request is one range
};
constexpr int kCand = 16;        // candidates; kWave / kCand = 4 lanes share one
constexpr int kPlanTiles = 256;  // requests staged in LDS at most

// A range's cost in tiles: its start (a tile of d = 64 is half as long) and the
// fp32 rows of its G heads and L queries, written and read once; at most ten.
__device__ inline int sp_range_cost(const SoftmaxPrefixArgs& a) {
  return min(10, (a.s.D == 128 ? 2 : 4) + a.s.Hq / a.s.Hkv * a.s.L / (a.s.dtype == 1 ? 16 : 32));
}

// Sum or maximum over the wave, in every lane: rotations within the rows of 16
// lanes, then exchanges of rows.  (Six shuffles through LDS took 0.3 us, and a
// plan and its use are several of these.)
template <typename Op>
__device__ inline int wave_all(int x, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));  // row_ror:8
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));
  auto f = [](int v) { return __builtin_bit_cast(float, v); };
  x = op(x, __builtin_bit_cast(int, xor16(f(x))));
  return op(x, __builtin_bit_cast(int, xor32(f(x))));
}
struct AddOp {
  __device__ int operator()(int a, int b) const { return a + b; }
};
struct MaxOp {
  __device__ int operator()(int a, int b) const { return max(a, b); }
};
struct MinOp {
  __device__ int operator()(int a, int b) const { return min(a, b); }
};
// Sum over the lanes up to this one.
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2, 3
  return x;
}

// tiles: LDS scratch of kPlanInts ints.  All threads of the workgroup; the
// first wave plans.  (The scratch is part of a tile buffer that is first written
// behind a later barrier: on its own it would cost d = 64 one of five workgroups
// on a CU.)
constexpr int kPlanInts = kPlanTiles + 2;
template <int WIN>
__device__ inline SpPlan sp_plan(const SoftmaxPrefixArgs& a, const SpCut& cut, int* tiles) {
  const int B = a.s.B, tid = threadIdx.x;
  static_assert(WIN < 2, "an 8-bit cache's plan is sp_even_plan");
  if (a.n_split == 1) return SpPlan{1 << 24, true};
  if (cut.c > 0) return SpPlan{cut.c, false};
  if (tid < kWave) {
    int total = 0, most = 0;
    const int end = B <= kPlanTiles ? (B + 15) & ~15 : B;  // (padded with empty requests)
    for (int b0 = tid; b0 < end; b0 += kWave) {
      const int nt = b0 < B ? sp_tiles<WIN>(a, b0) : 0;
      if (B <= kPlanTiles) tiles[b0] = nt;
      total += nt;
      most = max(most, nt);
    }
    total = __builtin_amdgcn_readfirstlane(wave_all(total, AddOp{}));
    most = __builtin_amdgcn_readfirstlane(wave_all(most, MaxOp{}));
    // (tiles: written and read by this wave)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    const int share = max(1, (total + cut.sat - 1) / cut.sat);
    const int cand = tid % kCand, sub = tid / kCand;
    // 1/4, 1/3, 1/2, 3/4, then from 1 on in steps of 1/16 to 1 1/2, 2, 4
    const int num = cand < 4 ? (cand == 0 ? 12 : cand == 1 ? 16 : cand == 2 ? 24 : 36)
                    : cand < 13 ? 48 + 3 * (cand - 4) : cand == 13 ? 96 : 192;
    int c = (int)(((long)share * num + 47) / 48);
    c = min(max(c, 4), kMaxRange / kTile);
    const int least = max(1, cut.limit / B);
    if (cand == kCand - 1) c = (most + least - 1) / least;
    // the candidate's ranges: x / c by a reciprocal, within one of it, so that
    // the correction leaves one too many at worst and never too few (c times the
    // quotient's error is below one for x up to 5 million); exact beyond
    const float rc = 1.0f / (float)c;
    auto ranges = [&](int x) {
      if (x >= 1 << 20) return (x + c - 1) / c;
      const int n = (int)((float)x * rc);
      return n + (n * c < x ? 1 : 0);
    };
    int sum = 0;
    if (B <= kPlanTiles) {
      for (int b0 = 4 * sub; b0 < end; b0 += 16) {
        const int4 x = *reinterpret_cast<const int4*>(tiles + b0);
        sum += ranges(x.x) + ranges(x.y) + ranges(x.z) + ranges(x.w);
      }
    } else {
      for (int b0 = sub; b0 < B; b0 += kWave / kCand) sum += ranges(sp_tiles<WIN>(a, b0));
    }
    static_assert(kCand == 16, "the lanes that share a candidate are a row apart");
    sum += __builtin_bit_cast(int, xor16(__builtin_bit_cast(float, sum)));
    sum += __builtin_bit_cast(int, xor32(__builtin_bit_cast(float, sum)));
    const int extra = sum > B ? sp_range_cost(a) : 0, longest = min(c, most) + extra;
    const int work = (min(total, 1 << 26) + sum * extra) * 11 / 10, rest = sum % cut.slots;
    int time = longest * cut.sat;
    if (sum > cut.slots)
      time = work + (rest > 0 ? time * (cut.slots - rest) / cut.slots : 0);
    else if (sum > cut.sat)
      time = max(longest * (cut.sat + (sum + cut.layer - 1) / cut.layer * cut.layer) / 2, work);
    const int cost = sum <= cut.limit ? time : cand == kCand - 1 ? 0x7ffffffe : 0x7fffffff;
    const int at = __builtin_ctzll(__ballot(cost == wave_all(cost, MinOp{})));
    const int pick = __builtin_amdgcn_readlane(c, at);
    if (tid == 0) {
      tiles[kPlanTiles] = pick;
      tiles[kPlanTiles + 1] = most <= pick;
    }
  }
  __syncthreads();
  return SpPlan{__builtin_amdgcn_readfirstlane(tiles[kPlanTiles]),
                __builtin_amdgcn_readfirstlane(tiles[kPlanTiles + 1]) != 0};
}

// The plan of an 8-bit cache's kernels: an even share of all tiles for B (n_split - 1) ranges, so
// that the requests' ranges, each rounded up, are at most B n_split.  Every wave works it out for
// itself, without LDS and without a barrier.
__device__ inline SpPlan sp_even_plan(const SoftmaxPrefixArgs& a, const SpCut& cut) {
  if (a.n_split == 1) return SpPlan{1 << 24, true};
  const int B = a.s.B;
  long sum = 0;
  int most = 0;
  for (int b = threadIdx.x % kWave; b < B; b += kWave) {
    const int nt = sp_tiles<2>(a, b);
    sum += nt;
    most = max(most, nt);
  }
  // (in two pieces: 2^31 tokens of each of many requests)
  const long total = ((long)__builtin_amdgcn_readfirstlane(wave_all((int)(sum >> 24), AddOp{})) << 24) +
                     __builtin_amdgcn_readfirstlane(wave_all((int)(sum & 0xffffff), AddOp{}));
  most = __builtin_amdgcn_readfirstlane(wave_all(most, MaxOp{}));
  const int share = cut.limit - B;
  const int c = (int)min(max((total + share - 1) / share, 1L), (long)kMaxRange / kTile);
  return SpPlan{c, most <= c};
}

// Ranges of a request of nt tiles.
__device__ inline int sp_ranges(const SpPlan& p, int nt) { return (nt + p.c - 1) / p.c; }

// Range number r of the plan: its request, its place there, how many ranges
// that request has and its keys lo .. hi-1 (with WIN: those of its tiles t0 ..
// t0 + nt - 1 that are visible).  b = -1: no such range.  Where every
// request is one range, that is request r; else the ranges of the requests
// before are summed, 64 requests at a time.  (Summed in every case, calls of
// many short requests paid for it: 4096 requests of 64 keys 907 us, now 377;
// 4096 of 32 at 8 KV heads of d = 64 584 us, now 141.)
struct SpRange {
  int b, s, n, lo, hi;
  int t0 = 0, nt = 0;  // WIN only
};
template <int WIN>
__device__ inline SpRange sp_share(const SoftmaxPrefixArgs& a, int b, int s, int n) {
  // an even share of the tiles: the first tiles % n ranges take one more
  const int keys = sp_keys<WIN>(a, b);
  const int tiles = WIN ? sp_tiles<WIN>(a, b) : (keys + kTile - 1) / kTile;
  const int each = tiles / n, more = tiles % n;
  const int t0 = s * each + min(s, more);
  if constexpr (WIN) {
    const SpSeen v = sp_seen<WIN>(a, b);
    const int nt = each + (s < more ? 1 : 0);
    return SpRange{b, s, n, v.tile(t0) * kTile, min((v.tile(t0 + nt - 1) + 1) * kTile, keys), t0, nt};
  } else {
    return SpRange{b, s, n, t0 * kTile, min((t0 + each + (s < more ? 1 : 0)) * kTile, keys)};
  }
}
template <int WIN>
__device__ inline SpRange sp_range(const SoftmaxPrefixArgs& a, const SpPlan& p, int r, int lane) {
  const int B = a.s.B;
  const SpRange none{-1, 0, 0, 0, 0};
  if constexpr (WIN) {
    if (p.whole) return r < B && sp_tiles<WIN>(a, r) > 0 ? sp_share<WIN>(a, r, 0, 1) : none;
  }
  if (p.whole) return r < B ? SpRange{r, 0, 1, 0, sp_keys<WIN>(a, r)} : none;
  int base = 0;
  for (int b0 = 0; b0 < B; b0 += kWave) {
    const int n = b0 + lane < B ? sp_ranges(p, sp_tiles<WIN>(a, b0 + lane)) : 0;
    const int end = wave_scan(n);
    const int all = __builtin_amdgcn_readlane(end, kWave - 1);
    if (r < base + all) {
      const int at = __builtin_ctzll(__ballot(r < base + end));
      const int nb = __builtin_amdgcn_readlane(n, at);
      return sp_share<WIN>(a, b0 + at, r - base - (__builtin_amdgcn_readlane(end, at) - nb), nb);
    }
    base += all;
  }
  return none;
}

// Partial results in the workspace, by range number r: rows of D floats
// [r][head][query], then (max, sum) pairs in the same order; at most n_split
// ranges per request on average.
__device__ inline size_t sp_row(const SoftmaxPrefixArgs& a, int r, int h, int i) {
  return ((size_t)r * a.s.Hq + h) * a.s.L + i;
}
template <int D>
__device__ inline float* sp_ml(const SoftmaxPrefixArgs& a) {
  return (float*)a.ws + (size_t)a.s.B * a.n_split * a.s.Hq * a.s.L * D;
}

// Four entries of a query's result: normalised into out, or as they are into
// the workspace where the request has more ranges.
template <typename T, int D>
__device__ inline void sp_put(const SoftmaxPrefixArgs& a, const SpRange& rg, int r, int h, int i, int at, const f32x4& o,
                              float den) {
  if (rg.n == 1) {
    const float inv = 1.0f / den;
    const float v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    store_out4<T>(a.out, (((size_t)rg.b * a.s.L + i) * a.s.Hq + h) * D + at, v, a.s.out_f32);
  } else {
    *reinterpret_cast<f32x4*>((float*)a.ws + sp_row(a, r, h, i) * D + at) = o;
  }
}
template <int D>
__device__ inline void sp_put_sum(const SoftmaxPrefixArgs& a, const SpRange& rg, int r, int h, int i, float m, float den) {
  if (rg.n == 1) return;
  float* wml = sp_ml<D>(a) + sp_row(a, r, h, i) * 2;
  wml[0] = m * 0.6931471805599453f;  // back to the natural log
  wml[1] = den;
}

// Where a range and KV head have several workgroups, for groups of heads: workgroup
// blockIdx.x is group hg of range and KV head `at`.  They read the same tiles, so
// they are eight workgroups apart, on one XCD (the last ranges, fewer than eight,
// as many apart as they are).
__device__ inline void sp_place(int groups, int& at, int& hg) {
  const int ats = gridDim.x / groups, at8 = blockIdx.x / (kNumXcd * groups) * kNumXcd, step = min(kNumXcd, ats - at8);
  const int in8 = blockIdx.x - at8 * groups;
  at = at8 + in8 % step;
  hg = in8 / step;
}

// Merge of the partial results of the requests that have several ranges.  A
// workgroup's unit of work is RPB rows of a (request, head), a thread 4
// columns of a row (16-byte loads); loads of several ranges are in flight at
// once, and up to four ranges are read before their weights are known.  A
// small merge is a chain of latencies (the plan, the maxima, the rows), so as
// many workgroups run as the chip holds (2048) and most take one unit: 32
// requests of 1024 keys 12.3 us, where 1024 workgroups of two units with
// the rows requested after the maxima took 13.7 us (8 requests: 7.2, now
// 5.4).
template <typename T, int D, int WIN = 0>
__global__ __launch_bounds__(256) void hyb_sp_combine_kernel(SoftmaxPrefixArgs a, SpCut cut) {
  constexpr int TPR = D / 4;              // threads per row
  constexpr int RPB = 256 / TPR;          // rows per unit
  SpPlan p;
  if constexpr (WIN == 2) {
    p = sp_even_plan(a, cut);
  } else {
    __shared__ alignas(16) int plan[kPlanInts];
    p = sp_plan<WIN>(a, cut, plan);
  }
  if (p.whole) return;  // every row is already written out
  const int Hq = a.s.Hq, L = a.s.L, lane = threadIdx.x & (kWave - 1);
  const int upb = (L + RPB - 1) / RPB;    // units of a (request, head)
  const float* wacc = (const float*)a.ws;
  const float* wml = sp_ml<D>(a);
  const size_t step = (size_t)Hq * L;  // rows from one range to the next
  for (int u = blockIdx.x; u < a.s.B * Hq * upb; u += gridDim.x) {
    const int bh = u / upb, b = bh / Hq, h = bh % Hq;
    const int n = sp_ranges(p, sp_tiles<WIN>(a, b));
    if (n == 1 || (WIN && n == 0)) continue;  // uniform: already written out (or no query)
    int base = 0;
    for (int b0 = lane; b0 < b; b0 += kWave) base += sp_ranges(p, sp_tiles<WIN>(a, b0));
    base = wave_all(base, AddOp{});
    const int i = u % upb * RPB + threadIdx.x / TPR, c = (threadIdx.x % TPR) * 4;
    if (i >= (WIN ? sp_block<WIN>(a, b) : L)) continue;  // (no barrier or exchange follows in this unit)
    const size_t row0 = sp_row(a, base, h, i);
    float M = -INFINITY;
    f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
    float den = 0.0f;
    if (n <= 4) {
      float2 ml[4];
      f32x4 x[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const size_t rr = row0 + min(s, n - 1) * step;
        ml[s] = *reinterpret_cast<const float2*>(wml + rr * 2);
        x[s] = *reinterpret_cast<const f32x4*>(wacc + rr * D + c);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) M = fmaxf(M, ml[s].x);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (s >= n || ml[s].x == -INFINITY) continue;
        const float wgt = expf(ml[s].x - M);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += wgt * x[s][e];
        den += wgt * ml[s].y;
      }
    } else {
#pragma unroll 8
      for (int s = 0; s < n; ++s) M = fmaxf(M, wml[(row0 + s * step) * 2]);
#pragma unroll 4
      for (int s = 0; s < n; ++s) {
        const size_t rr = row0 + s * step;
        const float ms = wml[rr * 2];
        if (ms == -INFINITY) continue;  // every score of the range is -inf
        const float wgt = expf(ms - M);
        const f32x4 x = *reinterpret_cast<const f32x4*>(wacc + rr * D + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += wgt * x[e];
        den += wgt * wml[rr * 2 + 1];
      }
    }
    const float o[4] = {num[0] / den, num[1] / den, num[2] / den, num[3] / den};
    store_out4<T>(a.out, (((size_t)b * L + i) * Hq + h) * D + c, o, a.s.out_f32);
  }
}

// Workgroups of a range kernel that the chip holds at once, by its LDS and
// registers as built.  Waves go to the four SIMDs in turn: 3, 5, 6 and 7 of them
// are counted as the next multiple of four (the odd ones seldom fit in between).
template <typename K>
static int sp_resident(K kernel, int waves) {
  int n = 0;
  const int w = waves <= 2 ? waves : (waves + 3) / 4 * 4;
  const hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kWave * w, 0);
  return 256 * (e == hipSuccess ? max(1, n) : 1);
}

template <typename K, typename A>
static hipError_t sp_launch(K kernel, int resident, int waves, bool ring, const A& a, hipStream_t st, SpCut* out,
                            int groups = 1) {
  const int ns = a.n_split, per = a.s.Hkv * groups;  // workgroups of a range
  SpCut cut;
  // Of the ring's workgroups two per CU, one with more than four waves, keep
  // the memory as busy as more do, three tiles of each in flight; the
  // register-staged kernel is bound by its waves' own chains.  (Two, or one, for
  // every kernel, also as what the chip holds, was right at d = 128 only: at
  // d = 64 up to five of the ring's workgroups fit: 32 requests of 1024 keys, 8
  // KV heads of one head, 26.7 us, now 19.2; 32 of 1 to 4096 keys at 16 KV heads,
  // paged, 115 and 77.)
  cut.slots = max(1, (waves > 4 ? min(resident, 256) : resident) / per);
  cut.sat = ring ? max(1, min(cut.slots, (waves > 4 ? 256 : 512) / per)) : cut.slots;
  // Ranges of a plan at most: three rounds, within the workspace, and at
  // least what the longest range allows.
  const int need = (int)(((long)a.max_seen + a.s.L + kMaxRange - 1) / kMaxRange);
  cut.limit = min(a.s.B * ns, max(a.s.B * need, 3 * cut.sat));
  cut.layer = max(1, 256 / per);
  // Where ranges of at most 512 keys of full-length requests fit one round,
  // the host cuts every request into those: there is little to gain from the
  // lengths, and working a plan out costs each kernel a few us (32 requests of
  // 1024 keys 43.8 against 37.4 us so, 8 of 4096 43.5 and 39.4, one of 8192
  // 32.7 and 28.8).
  const int tmax = (int)(((long)a.max_seen + a.s.L + kTile - 1) / kTile);
  const int even = (tmax + ns - 1) / ns;
  cut.c = 0;
  if ((long)a.s.B * ns <= cut.slots && even <= 16) {
    cut.c = even;
    cut.limit = a.s.B * ns;  // (full-length requests' ranges)
  }
  *out = cut;
  hipLaunchKernelGGL(kernel, dim3(per * cut.limit), dim3(kWave * waves), 0, st, a, cut);
  return hipGetLastError();
}

}  // namespace hyb
