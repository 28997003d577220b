// kv_q8.hip -- a paged KV cache in 8 bits: packed rows of new keys and values are
// quantised as they are written into its pages, and rows are read back.
//
// A scale block is scale_block consecutive rows of a page at one KV head.  For the
// block's new entries x, with m the largest finite |x|:
//   e    = the least whole number with m <= 448 2^e (448: the largest e4m3), >= -117
//   code = e4m3(x 2^-e), rounded to nearest even;  value = code 2^e
// Where the block goes on (its first rows hold earlier tokens), e is at least what it
// was, and where it grows the earlier codes c become e4m3(c 2^(old - e)).  A power of
// two as the scale keeps that exact but for codes that fall below 2^-6, costs e4m3 no
// precision (its step is relative) and makes every value exact in bf16.
//
// Bound: memory; each row is read once and its codes written once.  A job is a scale
// block's new rows at one head, of K or V: a wave holds 32 rows in registers between
// the maximum and the codes (blocks of more rows take a wave per 32, up to eight, and
// past 256 rows a second look at memory).  65536 tokens of 4 heads of d = 128, bf16, in blocks
// of 64: 37 us, 5.1 TB/s, what a copy reaches; with 64 rows per wave, fewer of which fit, 42,
// and 42 by stores that keep the codes in the caches.  Jobs are numbered so that request b's start
// at start_b / block + 2 b, which leaves every request room for the blocks it touches
// (its rows need not begin with a block) and needs no sums: a job finds its request by
// one look at the starts of 64 requests (two of 4096).
#include <algorithm>

#include "fp8.h"
#include "launch_cache.h"
#include "ragged.h"

namespace hyb {

constexpr int kQ8Rows = 32;   // rows that a wave holds (written)
constexpr int kQ8Waves = 8;   // of a workgroup that writes
constexpr int kQ8Readers = 4;

__host__ __device__ inline long q8_first_job(int start, int b, int shift) { return (long)(start >> shift) + 2L * b; }

// The rows lo .. lo + n - 1 (of k and v) that job `x` of blocks of 2^shift tokens
// covers, and where they are in the pools.
struct Q8Rows {
  int n = 0;       // none: nothing to do
  int src = 0;     // first row of k and v
  int at = 0;      // its place in the block
  size_t dst = 0;  // row of the pools where the block starts
  __device__ inline Q8Rows(const KvQ8Args& a, long x, int shift, int lane) {
    auto start = [&](int b) { return ragged_start(a.token_start, b, a.N); };
    const int b = ragged_find(a.B, x, lane, [&](int i) { return q8_first_job(start(i), i, shift); });
    const int s = start(b), e = start(b + 1), cap = a.max_pages << a.page_shift;
    const long p0 = min(max(a.first[b], 0), cap), p1 = min(p0 + max(e - s, 0), (long)cap);
    const long j0 = ((p0 >> shift) + x - q8_first_job(s, b, shift)) << shift;
    const long from = max(p0, j0), to = min(p1, j0 + (1L << shift));
    if (from >= to) return;
    const int page = a.page_table[(size_t)b * a.max_pages + (j0 >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) return;
    n = (int)(to - from);
    src = s + (int)(from - p0);
    at = (int)(from - j0);
    dst = ((size_t)page << a.page_shift) + (j0 & ((1L << a.page_shift) - 1));
  }
};

// Eight entries of a row.
template <typename T>
struct Q8Piece;
template <>
struct Q8Piece<bf16> {
  bf16x8 x;
  __device__ inline void load(const bf16* p) { x = *reinterpret_cast<const bf16x8*>(p); }
  __device__ inline float operator[](int e) const { return (float)x[e]; }
};
template <>
struct Q8Piece<float> {
  f32x4 a, b;
  __device__ inline void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ inline float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
};

// Largest of x over the wave, in every lane.
__device__ inline int q8_wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));  // row_ror:8
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));
  auto f = [](int v) { return __builtin_bit_cast(float, v); };
  x = max(x, __builtin_bit_cast(int, xor16(f(x))));
  return max(x, __builtin_bit_cast(int, xor32(f(x))));
}

// W waves share a job.  Codes are stored past the caches: a call writes more than it reads again.
template <typename T, int D, int W>
__global__ __launch_bounds__(kWave* kQ8Waves) void hyb_kv_q8_write_kernel(KvQ8Args a, long jobs) {
  constexpr int LPR = D / 8;           // lanes per row
  constexpr int RPI = kWave / LPR;     // rows per load
  constexpr int NL = kQ8Rows / RPI;    // loads that a wave holds
  __shared__ int most[kQ8Waves];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int w = wave % W;
  const long job = min((long)blockIdx.x * (kQ8Waves / W) + wave / W, jobs);  // (behind the last: nothing)
  const int g = (int)(job % a.Hkv), kv = (int)(job / a.Hkv & 1);
  Q8Rows r(a, job / a.Hkv >> 1, a.sb_shift, lane);
  if (job == jobs) r.n = 0;
  if (W == 1 && r.n == 0) return;  // (else at the barrier)
  const long stride = kv ? a.v_stride : a.k_stride;
  const T* src = (const T*)(kv ? a.v : a.k) + r.src * stride + (long)g * D + lane % LPR * 8;
  uint8_t* const pool = kv ? a.v_pages : a.k_pages;
  uint8_t* const scale = (kv ? a.v_scales : a.k_scales) + (r.dst >> a.sb_shift) * a.Hkv + g;
  const int old = r.n > 0 && r.at > 0 ? *scale : 0;
  Q8Piece<T> x[NL];
  int m = 0;
  // This wave's rows, 32 at a time: w, w + W, ..; those past the last are the last again.
  auto load = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NL; ++u)
      if (c0 + u * RPI < r.n) x[u].load(src + min(c0 + u * RPI + lane / LPR, r.n - 1) * stride);
  };
  int last = -1;
  for (int c0 = w * kQ8Rows; c0 < r.n; c0 += W * kQ8Rows) {
    load(c0);
    last = c0;
#pragma unroll
    for (int u = 0; u < NL; ++u)
      if (c0 + u * RPI < r.n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int bits = __builtin_bit_cast(int, x[u][e]) & 0x7fffffff;
          m = max(m, bits < 0x7f800000 ? bits : 0);
        }
      }
  }
  m = q8_wave_max(m);
  if constexpr (W > 1) {
    if (lane == 0) most[wave] = m;
    __syncthreads();
    if (r.n == 0) return;
#pragma unroll
    for (int i = 0; i < W; ++i) m = max(m, most[wave - w + i]);
  }
  const int byte = max(scale_byte(__builtin_amdgcn_readfirstlane(m)), old);
  if (w == 0 && lane == 0) *scale = (uint8_t)byte;
  if (r.at > 0 && old < byte) {  // the scale grows: the block's earlier rows (16 codes per lane)
    constexpr int LPC = D / 16;
    const float f = scale_of(max(old - byte + 127, 0));
    for (int i = (w * kWave + lane) / LPC; i < r.at; i += W * kWave / LPC) {
      uint4* const p = reinterpret_cast<uint4*>(pool + ((r.dst + i) * a.Hkv + g) * D + lane % LPC * 16);
      const uint4 c = *p;
      auto fewer = [f](uint32_t c4) {
        const f32x4 y = fp8_f32(c4, 1.0f);
        return fp8_codes(y[0], y[1], y[2], y[3], f);
      };
      *p = uint4{fewer(c.x), fewer(c.y), fewer(c.z), fewer(c.w)};
    }
  }
  const float f = scale_of(254 - min(byte, 254));  // (255, NaN, stays, whatever the codes)
  for (int c0 = w * kQ8Rows; c0 < r.n; c0 += W * kQ8Rows) {
    if (c0 != last || c0 != w * kQ8Rows) load(c0);  // (held where the wave has no more)
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const int i = c0 + u * RPI + lane / LPR;
      if (c0 + u * RPI < r.n && i < r.n) {
        const uint2 c = {fp8_codes(x[u][0], x[u][1], x[u][2], x[u][3], f),
                         fp8_codes(x[u][4], x[u][5], x[u][6], x[u][7], f)};
        __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, c), reinterpret_cast<uint64_t*>(
            pool + ((r.dst + r.at + i) * a.Hkv + g) * D + lane % LPR * 8));
      }
    }
  }
}

// Reading: a job is at most 64 rows of a scale block at one head, of K or V.  (64000 tokens of 4
// heads of d = 128 into bf16: 31 us, 6.4 TB/s; 43 where the rows are stored by way of the caches.)
template <typename T, int D>
__global__ __launch_bounds__(kWave* kQ8Readers) void hyb_kv_q8_read_kernel(KvQ8Args a, long jobs, int shift) {
  constexpr int LPR = D / 8, RPI = kWave / LPR, NL = 64 / RPI;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long job = (long)blockIdx.x * kQ8Readers + wave;
  if (job >= jobs) return;
  const int g = (int)(job % a.Hkv), kv = (int)(job / a.Hkv & 1);
  const Q8Rows r(a, job / a.Hkv >> 1, shift, lane);
  if (r.n == 0) return;
  const long stride = kv ? a.v_stride : a.k_stride;
  T* dst = (T*)(kv ? a.v : a.k) + r.src * stride + (long)g * D + lane % LPR * 8;
  const uint8_t* pool = (kv ? a.v_pages : a.k_pages) + ((r.dst + r.at) * a.Hkv + g) * D + lane % LPR * 8;
  const float f = scale_of((kv ? a.v_scales : a.k_scales)[(r.dst >> a.sb_shift) * a.Hkv + g]);
  uint2 c[NL];
#pragma unroll
  for (int u = 0; u < NL; ++u)
    if (u * RPI < r.n)
      c[u] = *reinterpret_cast<const uint2*>(pool + (size_t)min(u * RPI + lane / LPR, r.n - 1) * a.Hkv * D);
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    const int i = u * RPI + lane / LPR;
    if (u * RPI < r.n && i < r.n) {
      if constexpr (sizeof(T) == 2) {
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, fp8_bf16(c[u].x, c[u].y, f)),
                                    reinterpret_cast<u32x4*>(dst + i * stride));
      } else {
        __builtin_nontemporal_store(fp8_f32(c[u].x, f), reinterpret_cast<f32x4*>(dst + i * stride));
        __builtin_nontemporal_store(fp8_f32(c[u].y, f), reinterpret_cast<f32x4*>(dst + i * stride + 4));
      }
    }
  }
}

// Jobs for blocks of 2^shift tokens.
static long q8_jobs(const KvQ8Args& a, int shift) { return q8_first_job(a.N, a.B, shift) * 2 * a.Hkv; }
static int q8_read_shift(const KvQ8Args& a) { return std::min(a.sb_shift, 6); }

// Waves of a job.
static int q8_write_waves(const KvQ8Args& a) { return std::min(kQ8Waves, std::max(1, (1 << a.sb_shift) / kQ8Rows)); }

double kv_q8_threads(const KvQ8Args& a) {
  return kWave * (kQ8Waves + std::max((double)q8_jobs(a, q8_read_shift(a)), (double)q8_jobs(a, a.sb_shift) * q8_write_waves(a)));
}

template <typename T, int D>
static hipError_t q8_write_go(const KvQ8Args& a, hipStream_t st) {
  const long jobs = q8_jobs(a, a.sb_shift);
  const int waves = q8_write_waves(a);
  const dim3 grid((unsigned)((jobs * waves + kQ8Waves - 1) / kQ8Waves)), block(kWave * kQ8Waves);
  switch (waves) {
    case 1: hipLaunchKernelGGL((hyb_kv_q8_write_kernel<T, D, 1>), grid, block, 0, st, a, jobs); break;
    case 2: hipLaunchKernelGGL((hyb_kv_q8_write_kernel<T, D, 2>), grid, block, 0, st, a, jobs); break;
    case 4: hipLaunchKernelGGL((hyb_kv_q8_write_kernel<T, D, 4>), grid, block, 0, st, a, jobs); break;
    default: hipLaunchKernelGGL((hyb_kv_q8_write_kernel<T, D, 8>), grid, block, 0, st, a, jobs);
  }
  return hipGetLastError();
}
template <typename T, int D>
static hipError_t q8_read_go(const KvQ8Args& a, hipStream_t st) {
  const int shift = q8_read_shift(a);
  const long jobs = q8_jobs(a, shift);
  hipLaunchKernelGGL((hyb_kv_q8_read_kernel<T, D>), dim3((unsigned)((jobs + kQ8Readers - 1) / kQ8Readers)),
                     dim3(kWave * kQ8Readers), 0, st, a, jobs, shift);
  return hipGetLastError();
}

hipError_t launch_kv_q8_write(const KvQ8Args& a, hipStream_t st) {
  if (a.dtype == 1) return a.D == 64 ? q8_write_go<bf16, 64>(a, st) : q8_write_go<bf16, 128>(a, st);
  return a.D == 64 ? q8_write_go<float, 64>(a, st) : q8_write_go<float, 128>(a, st);
}
hipError_t launch_kv_q8_read(const KvQ8Args& a, hipStream_t st) {
  if (a.dtype == 1) return a.D == 64 ? q8_read_go<bf16, 64>(a, st) : q8_read_go<bf16, 128>(a, st);
  return a.D == 64 ? q8_read_go<float, 64>(a, st) : q8_read_go<float, 128>(a, st);
}

}  // namespace hyb
