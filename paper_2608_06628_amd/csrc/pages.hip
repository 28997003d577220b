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
// workgroups need no order among them.  (64 requests of a block each 5 us; 512 of up to
// 4096 tokens, a million in all, 8 us.)
#include <algorithm>

#include "device.h"
#include "launch.h"

namespace hyb {

constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 4;  // neighbouring tokens of a thread, found by one search

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

// Sums that stay at 2^31 - 1 (of terms that are not negative, so the order of
// the additions does not matter).
__device__ inline int plan_add(int a, int b) { return __builtin_elementwise_add_sat(a, b); }
// Sum over the lanes up to this one, by shifts within and broadcasts between the
// rows of 16 lanes.
__device__ inline int plan_scan(int x) {
  x = plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));   // row_shr:1
  x = plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
  x = plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
  x = plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
  x = plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1, 3
  return plan_add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2, 3
}

__global__ __launch_bounds__(kPlanThreads) void hyb_pages_plan_kernel(PagesArgs a) {
  // per request the first of its tokens and of its new pages (B + 1 entries:
  // the totals last), then its cached tokens
  extern __shared__ int sums[];
  __shared__ int carry[2][kPlanThreads / kWave];
  const int B = a.B, tid = threadIdx.x, wave = tid / kWave;
  const int page = 1 << a.page_shift;
  const long cap = (long)a.max_pages << a.page_shift;
  int* const start = sums;
  int* const first = sums + B + 1;
  int* const cached = first + B + 1;
  auto held = [&](int p) { return (int)(((long)p + page - 1) >> a.page_shift); };

  // Running sums: a thread takes `each` neighbouring requests (one where they fit).
  const int each = (B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(tid * each, B), b1 = min(b0 + each, B);
  int nt = 0, np = 0;
  for (int b = b0; b < b1; ++b) {
    const int p = min(max(a.prefix_len[b], 0), (int)cap), n = max(a.new_len[b], 0);
    const int need = (int)((min((long)p + n, cap) + page - 1) >> a.page_shift) - held(p);
    // (the thread's own sums for now)
    cached[b] = p;
    start[b] = nt;
    first[b] = np;
    nt = plan_add(nt, n);
    np = plan_add(np, need);
  }
  const int it = plan_scan(nt), ip = plan_scan(np);
  if (tid % kWave == kWave - 1) carry[0][wave] = it, carry[1][wave] = ip;
  // what the lanes before hold (a saturated sum cannot be taken back by its
  // last term)
  int et = __builtin_amdgcn_update_dpp(0, it, 0x138, 0xf, 0xf, false);  // wave_shr:1
  int ep = __builtin_amdgcn_update_dpp(0, ip, 0x138, 0xf, 0xf, false);
  __syncthreads();
  int tokens = 0, pages = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) et = plan_add(et, carry[0][w]), ep = plan_add(ep, carry[1][w]);
    tokens = plan_add(tokens, carry[0][w]);
    pages = plan_add(pages, carry[1][w]);
  }
  for (int b = b0; b < b1; ++b) {
    start[b] = plan_add(start[b], et);
    first[b] = plan_add(first[b], ep);
  }
  if (tid == 0) {
    start[B] = tokens;
    first[B] = pages;
  }
  __syncthreads();
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
    const int e = held(cached[b]) + ((int)i - first[b]);
    a.page_table[(size_t)b * a.max_pages + e] = i < a.n_free ? a.free_pages[i] : -1;
  }
  // The tokens' slots and positions.
  for (long t0 = ((long)blockIdx.x * kPlanThreads + tid) * kPlanTokens; t0 < a.max_tokens;
       t0 += (long)gridDim.x * kPlanThreads * kPlanTokens) {
    int slot[kPlanTokens], pos[kPlanTokens];
    int b = t0 < tokens ? plan_find(start, B, (int)t0) : B - 1;
#pragma unroll
    for (int u = 0; u < kPlanTokens; ++u) {
      const long t = t0 + u;
      slot[u] = -1;
      pos[u] = 0;
      if (t >= tokens) continue;
      while (b + 1 < B && start[b + 1] <= t) ++b;
      const int p = cached[b];
      const long x = (long)p + (t - start[b]);
      pos[u] = (int)min(x, 0x7fffffffL);
      if (x >= cap) continue;
      const int e = (int)(x >> a.page_shift), h = held(p);
      const long i = (long)first[b] + (e - h);
      long pg = -1;
      if (e < h)
        pg = a.page_table[(size_t)b * a.max_pages + e];
      else if (i < a.n_free)
        pg = a.free_pages[i];
      const long row = (pg << a.page_shift) + (x & (page - 1));
      slot[u] = pg < 0 || row > 0x7fffffffL ? -1 : (int)row;
    }
    if (t0 + kPlanTokens <= a.max_tokens) {
      *reinterpret_cast<int4*>(a.slots + t0) = int4{slot[0], slot[1], slot[2], slot[3]};
      *reinterpret_cast<int4*>(a.positions + t0) = int4{pos[0], pos[1], pos[2], pos[3]};
    } else {
      for (int u = 0; u < (int)(a.max_tokens - t0); ++u) {
        a.slots[t0 + u] = slot[u];
        a.positions[t0 + u] = pos[u];
      }
    }
  }
}

hipError_t launch_pages_plan(const PagesArgs& a, hipStream_t st) {
  // Workgroups for the tokens; the table's entries are fewer, and taken by the
  // same ones.
  const long per = kPlanThreads * kPlanTokens;
  const unsigned grid = (unsigned)std::min<long>(std::max<long>(1, (a.max_tokens + per - 1) / per), 2048);
  hipLaunchKernelGGL(hyb_pages_plan_kernel, dim3(grid), dim3(kPlanThreads), (3 * a.B + 2) * sizeof(int), st, a);
  return hipGetLastError();
}

}  // namespace hyb
