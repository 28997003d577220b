// launch_cache.h -- internal interface between the C-ABI layer (api.cpp) and the
// kernels of the 8-bit KV cache.  Arguments arrive here already validated.
#pragma once

#include "launch.h"

namespace hyb {

// Rows of packed tokens into (kv_q8.hip: write) or out of (read) the pools of an
// 8-bit paged cache.  Request b's tokens are rows token_start[b] .. token_start[b + 1]
// - 1 of k and v and tokens first[b] .. of its cache.
struct KvQ8Args {
  int N, B, Hkv, D, dtype;
  int max_pages, n_pages, page_shift, sb_shift;  // log2 of a page's and a scale block's tokens
  long k_stride, v_stride;                       // elements from a token's row to the next
  void *k, *v;                                   // write: only read
  const int32_t *page_table, *first, *token_start;
  uint8_t *k_pages, *v_pages;    // [n_pages][page][Hkv][D] e4m3
  uint8_t *k_scales, *v_scales;  // [n_pages][page / block][Hkv] exponent + 127
};

// Softmax over such a cache (softmax_q8.hip): k_cache and v_cache of the base are the
// pools' codes, window >= 0.
struct SoftmaxQ8Args : SoftmaxPrefixArgs {
  const uint8_t *k_scales, *v_scales;
  int sb_shift;
};

hipError_t launch_kv_q8_write(const KvQ8Args& a, hipStream_t st);
hipError_t launch_kv_q8_read(const KvQ8Args& a, hipStream_t st);
double kv_q8_threads(const KvQ8Args& a);  // of the larger grid
hipError_t launch_softmax_q8(const SoftmaxQ8Args& a, hipStream_t st);
double softmax_q8_threads(const SoftmaxQ8Args& a);
// Ranges per request at most, for max_seen cached tokens, the tokens that fill the
// cache's last tile up among them.
int softmax_q8_splits(const Shape& s, int max_seen);

}  // namespace hyb
