// pages.hip -- pages and cache rows of a batch's new tokens, from the
// requests' lengths on the device: what a serving engine needs before it can
// write keys and values into a paged cache and read them back, without waiting
// for the lengths on the host.
//
//   need_b  = ceil(min(p_b + n_b, cap) / page) - ceil(p_b / page)
//   first_b = sum of need over the requests before b
//   entry ceil(p_b / page) + i of request b  <-  free_pages[first_b + i]
//   slot of token t of request b = page of entry (p_b + t) / page, row
//   (p_b + t) % page
//
// Bound: a chain of latencies (the lengths, their running sums, a search, one
// gather), and for prompts the stores of slots and positions.  One launch:
// every workgroup sums the lengths of all requests itself (they come from
// the caches, and a second launch would cost more than the sums) and takes a
// share of the tokens and of the table's new entries, each found by a binary
// search of the running sums in LDS.  Entries of the table that this call
// writes are never read by it: their pages come from free_pages, so the
// workgroups need no order among them.
#include <algorithm>

#include "device.h"
#include "launch.h"

namespace hyb {

constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 4;  // tokens of a thread and round

// Index of the last of sums[0 .. n] (not falling, sums[0] = 0) that is <= x,
// below n.
__device__ inline int plan_find(const int* sums, int n, int x) {
  int lo = 0, hi = n;  // sums[lo] <= x < sums[hi], or hi = n
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void hyb_pages_plan_kernel(PagesArgs a) {
  extern __shared__ int sums[];  // token starts [B + 1], then page starts [B + 1]
  __shared__ long carry[2][kPlanThreads / kWave];
  const int B = a.B, tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int page = 1 << a.page_shift;
  const long cap = (long)a.max_pages << a.page_shift;
  int* const start = sums;
  int* const first = sums + B + 1;
  auto prefix = [&](int b) { return (int)min((long)max(a.prefix_len[b], 0), cap); };
  auto held = [&](int p) { return (int)(((long)p + page - 1) >> a.page_shift); };
  auto saturated = [](long x) { return (int)min(x, 0x7fffffffL); };

  // Running sums: a thread takes `each` neighbouring requests.
  const int each = (B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(tid * each, B), b1 = min(b0 + each, B);
  long nt = 0, np = 0;
  for (int b = b0; b < b1; ++b) {
    const int p = prefix(b), n = max(a.new_len[b], 0);
    nt += n;
    np += ((min((long)p + n, cap) + page - 1) >> a.page_shift) - held(p);
  }
  long it = nt, ip = np;  // inclusive over the wave
  for (int o = 1; o < kWave; o <<= 1) {
    const long x = __shfl_up(it, o), y = __shfl_up(ip, o);
    if (lane >= o) it += x, ip += y;
  }
  if (lane == kWave - 1) carry[0][wave] = it, carry[1][wave] = ip;
  __syncthreads();
  long et = it - nt, ep = ip - np;
  for (int w = 0; w < wave; ++w) et += carry[0][w], ep += carry[1][w];
  for (int b = b0; b < b1; ++b) {
    const int p = prefix(b), n = max(a.new_len[b], 0);
    start[b] = saturated(et);
    first[b] = saturated(ep);
    et += n;
    ep += ((min((long)p + n, cap) + page - 1) >> a.page_shift) - held(p);
  }
  long all_t = 0, all_p = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) all_t += carry[0][w], all_p += carry[1][w];
  if (tid == 0) {
    start[B] = saturated(all_t);
    first[B] = saturated(all_p);
  }
  __syncthreads();
  const int tokens = start[B], pages = first[B];
  if (blockIdx.x == 0) {
    for (int b = tid; b <= B; b += kPlanThreads) a.token_start[b] = start[b];
    if (tid == 0) {
      a.counts[0] = min(pages, a.n_free);
      a.counts[1] = max(pages - a.n_free, 0);
    }
  }
  // The table's new entries.
  for (long i = (long)blockIdx.x * kPlanThreads + tid; i < pages; i += (long)gridDim.x * kPlanThreads) {
    const int b = plan_find(first, B, (int)i);
    const int e = held(prefix(b)) + ((int)i - first[b]);
    a.page_table[(size_t)b * a.max_pages + e] = i < a.n_free ? a.free_pages[i] : -1;
  }
  // The tokens' slots and positions.
  for (long t0 = (long)blockIdx.x * kPlanThreads * kPlanTokens; t0 < a.max_tokens;
       t0 += (long)gridDim.x * kPlanThreads * kPlanTokens) {
#pragma unroll
    for (int u = 0; u < kPlanTokens; ++u) {
      const long t = t0 + u * kPlanThreads + tid;
      if (t >= a.max_tokens) break;
      long slot = -1, pos = 0;
      if (t < tokens) {
        const int b = plan_find(start, B, (int)t);
        const int p = prefix(b);
        pos = (long)p + (t - start[b]);
        if (pos < cap) {
          const int e = (int)(pos >> a.page_shift), h = held(p);
          long pg;
          if (e < h) {
            pg = a.page_table[(size_t)b * a.max_pages + e];
          } else {
            const long i = (long)first[b] + (e - h);
            pg = i < a.n_free ? a.free_pages[i] : -1;
          }
          slot = pg < 0 ? -1 : (pg << a.page_shift) + (pos & (page - 1));
          if (slot > 0x7fffffffL) slot = -1;
        }
      }
      a.slots[t] = (int)slot;
      a.positions[t] = saturated(pos);
    }
  }
}

hipError_t launch_pages_plan(const PagesArgs& a, hipStream_t st) {
  // Workgroups for the tokens; the table's entries are fewer (a page of 16
  // rows and more), and taken by the same ones.
  const long per = kPlanThreads * kPlanTokens;
  const unsigned grid = (unsigned)std::min<long>(std::max<long>(1, (a.max_tokens + per - 1) / per), 2048);
  hipLaunchKernelGGL(hyb_pages_plan_kernel, dim3(grid), dim3(kPlanThreads), 2 * (a.B + 1) * sizeof(int), st, a);
  return hipGetLastError();
}

}  // namespace hyb
