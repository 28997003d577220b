// rope.hip -- per-head RMS norm of queries and keys with the rotation by
// position in the same pass, the same with keys and values written into a
// paged cache, and the gradient: what stands between the projections and
// every attention layer here.
//
//   forward   r = 1 / sqrt(mean(x^2) + eps),  n = x r w
//             (a, b) -> c (a cos t - b sin t, b cos t + a sin t) for every
//             rotated pair (a, b) of n, t = position * inv_freq[i]
//   backward  u = c R(-t) g,  dw = sum u x r,
//             dx = r (u w - x r mean(u w x r))
//
// Bound: HBM.  A row (one head of one token) is read once and written once;
// everything between stays in the registers of D / 8 lanes, 8 entries each: a
// lane holds two 4-entry pieces that contain both members of its pairs in
// either layout (half: entries 4r.. and rot/2 + 4r..; interleaved: 8r.. and
// 8r + 4..), so the rotation needs no exchange and the norm's mean is a
// reduction over 8 or 16 neighbouring lanes, four DPP additions.  A wave takes
// 64 / (D / 8) heads at a time.  The angles depend on the token and the lane
// only, so a wave computes them once and keeps them for all the heads it
// handles of that token (the angle itself in 64 bits, because a position of a
// million times a frequency leaves an fp32 angle 0.06 off; its sine and cosine
// in 32).
//
// Measured, 16 and 4 heads of d = 128, bf16: 65536 tokens 127 us a call, one after the other
// (5.3 TB/s; fp32, 16384 tokens, 64); the kernels alone, under a trace: 64 tokens into pages 4 us,
// gradient of 16384 tokens 44 us (5.7 TB/s), and 5 for the weights' sums.
#include <algorithm>
#include <type_traits>

#include "device.h"
#include "launch.h"

namespace hyb {

// Sum over the LPR (8 or 16) neighbouring lanes that share a row, in all of
// them: x with lane ^ 1, lane ^ 2 (quad permutations), 7 - i within 8 lanes
// and 15 - i within 16 (mirrors: after the quads agree any lane of the other
// quad will do).
template <int LPR>
__device__ inline float row_sum(float x) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x += dpp(x, std::integral_constant<int, 0xb1>{});   // quad_perm 1,0,3,2
  x += dpp(x, std::integral_constant<int, 0x4e>{});   // quad_perm 2,3,0,1
  x += dpp(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LPR == 16) x += dpp(x, std::integral_constant<int, 0x140>{});  // row_mirror
  return x;
}

// 8 entries of a row as two pieces of four, at p0 and p1: as loaded (so that a
// load can be on its way while others are used), and as fp32.
template <typename T>
struct Pieces {
  typedef T piece_t __attribute__((ext_vector_type(4)));
  piece_t a = {}, b = {};
  __device__ inline void load(const T* p0, const T* p1) {
    a = *reinterpret_cast<const piece_t*>(p0);
    b = *reinterpret_cast<const piece_t*>(p1);
  }
  __device__ inline void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)a[i], x[4 + i] = (float)b[i];
  }
};
template <typename T>
__device__ inline void load_pieces(const T* p0, const T* p1, float (&x)[8]) {
  Pieces<T> p;
  p.load(p0, p1);
  p.get(x);
}
template <typename T>
__device__ inline void store_pieces(T* p0, T* p1, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(p0) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p1) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    *reinterpret_cast<bf16x4*>(p0) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
    *reinterpret_cast<bf16x4*>(p1) = bf16x4{(bf16)x[4], (bf16)x[5], (bf16)x[6], (bf16)x[7]};
  }
}

// What a lane keeps of a token's rotation: whether its entries are rotated at
// all, where its two pieces are, and the cosines and sines (times the scale)
// of its four pairs: entries (i, 4 + i) of the lane, or (2i, 2i + 1) with
// INTER (pairs side by side).
template <bool INTER>
struct Turn {
  bool rot;
  int e0, e1;
  float c[4], s[4];
  double freq[4];  // turns per position

  __device__ inline Turn(const RopeArgs& a, int r) {
    rot = r < a.rot / 8;
    const bool apart = !INTER && rot;  // the pieces are half the rotated part apart
    e0 = apart ? 4 * r : 8 * r;
    e1 = apart ? a.rot / 2 + 4 * r : 8 * r + 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) freq[i] = rot ? a.inv_freq[4 * r + i] * 0.15915494309189535 : 0.0;
  }
  // The angles in turns, reduced to half a turn in 64 bits; their sines and
  // cosines in 32 (the reduced angle's rounding moves it by at most 2^-26 of a turn,
  // 9e-8 rad, an fp32 rounding).
  __device__ inline void at(int pos, float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double turns = (double)pos * freq[i];
      sincospif(2.0f * (float)(turns - rint(turns)), &s[i], &c[i]);
      c[i] *= scale;
      s[i] *= scale;
    }
  }
  // Rotates the lane's entries, by the angles or (INV) back.
  template <bool INV>
  __device__ inline void apply(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      constexpr int kStep = INTER ? 2 : 1, kOther = INTER ? 1 : 4;
      const float a = x[kStep * i], b = x[kStep * i + kOther], sn = INV ? -s[i] : s[i];
      x[kStep * i] = rot ? a * c[i] - b * sn : a;
      x[kStep * i + kOther] = rot ? b * c[i] + a * sn : b;
    }
  }
};

// Work units: a token and `per` groups of heads of it (a group is what a wave
// takes at a time).  Few tokens take a group per wave, so that the call is one
// chain of loads long; many tokens take all groups of a token, so that its
// angles are computed once.
struct RopeUnits {
  int groups, per, parts;  // groups of a token, of a unit; units of a token
  long n;
};
static RopeUnits rope_units(long tokens, int heads, int heads_per_group, long waves) {
  RopeUnits u;
  u.groups = (heads + heads_per_group - 1) / heads_per_group;
  u.per = (int)std::min<long>(u.groups, std::max<long>(1, tokens * u.groups / waves));
  u.parts = (u.groups + u.per - 1) / u.per;
  u.per = (u.groups + u.parts - 1) / u.parts;
  u.n = tokens * u.parts;
  return u;
}

constexpr int kRopeWaves = 4;  // waves of a workgroup

// Heads are numbered through: the query heads, the KV heads' keys, and with
// PAGED their values.
template <typename T, typename O, int D, bool INTER, bool PAGED>
__global__ __launch_bounds__(kWave* kRopeWaves) void hyb_rope_kernel(RopeArgs a, RopeUnits u) {
  constexpr int LPR = D / 8, HPG = kWave / LPR;
  const int lane = threadIdx.x & (kWave - 1), r = lane % LPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = a.Hq + (PAGED ? 2 : 1) * a.Hkv;
  Turn<INTER> t(a, r);
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.0f;
  if (a.wq) load_pieces((const T*)a.wq + t.e0, (const T*)a.wq + t.e1, wq);
  if (a.wk) load_pieces((const T*)a.wk + t.e0, (const T*)a.wk + t.e1, wk);
  for (long un = (long)blockIdx.x * kRopeWaves + wave; un < u.n; un += (long)gridDim.x * kRopeWaves) {
    const long tok = un / u.parts;
    const int g0 = (int)(un - tok * u.parts) * u.per, g1 = min(g0 + u.per, u.groups);
    long slot = -1;
    if constexpr (PAGED) {
      slot = a.slots[tok];
      if (slot >= a.n_rows) slot = -1;
    }
    const int pos = a.positions[tok];
    Pieces<T> next;
    auto load = [&](int gr) __attribute__((always_inline)) {
      const int h = gr * HPG + lane / LPR;
      const bool isq = h < a.Hq, isv = PAGED && h >= a.Hq + a.Hkv;
      const T* row = isq   ? (const T*)a.q + tok * a.q_stride + h * D
                     : isv ? (const T*)a.v + tok * a.v_stride + (h - a.Hq - a.Hkv) * D
                           : (const T*)a.k + tok * a.k_stride + (h - a.Hq) * D;
      if (h < heads) next.load(row + t.e0, row + t.e1);
    };
    load(g0);
    t.at(pos, a.rot_scale);
    for (int gr = g0; gr < g1; ++gr) {
      const int h = gr * HPG + lane / LPR;
      const bool live = h < heads, isq = h < a.Hq, isv = PAGED && h >= a.Hq + a.Hkv;
      const int hk = isv ? h - a.Hq - a.Hkv : h - a.Hq;
      float x[8];
      next.get(x);
      if (gr + 1 < g1) load(gr + 1);
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
      ss = row_sum<LPR>(ss);
      if (!live) continue;
      if (!isv) {
        if (isq ? a.wq != nullptr : a.wk != nullptr) {
          const float rs = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= rs * (isq ? wq[i] : wk[i]);
        }
        t.template apply<false>(x);
        O* o = isq ? (O*)a.q_out + tok * a.q_out_stride + h * D
               : a.k_out ? (O*)a.k_out + tok * a.k_out_stride + hk * D
                         : nullptr;
        if (o) store_pieces(o + t.e0, o + t.e1, x);
      }
      if (PAGED && !isq && slot >= 0) {
        T* o = (T*)(isv ? a.v_pages : a.k_pages) + (slot * a.Hkv + hk) * D;
        store_pieces(o + t.e0, o + t.e1, x);
      }
    }
  }
}

// The gradient.  Besides dx a lane sums u x r of its 8 entries over the rows
// it handles, queries and keys apart; the lanes and waves of a workgroup are
// joined in LDS and leave one partial row of 2 D floats in the workspace, which
// a second kernel adds up in order.  The grid follows from the sizes alone, so
// the sums come out the same every time.
template <typename T, typename G, typename O, int D, bool INTER>
__global__ __launch_bounds__(kWave* kRopeWaves) void hyb_rope_backward_kernel(RopeArgs a, RopeUnits u) {
  constexpr int LPR = D / 8, HPG = kWave / LPR;
  const int lane = threadIdx.x & (kWave - 1), r = lane % LPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = a.Hq + a.Hkv;
  Turn<INTER> t(a, r);
  float wq[8], wk[8], sq[8] = {}, sk[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.0f;
  if (a.wq) load_pieces((const T*)a.wq + t.e0, (const T*)a.wq + t.e1, wq);
  if (a.wk) load_pieces((const T*)a.wk + t.e0, (const T*)a.wk + t.e1, wk);
  for (long un = (long)blockIdx.x * kRopeWaves + wave; un < u.n; un += (long)gridDim.x * kRopeWaves) {
    const long tok = un / u.parts;
    const int g0 = (int)(un - tok * u.parts) * u.per, g1 = min(g0 + u.per, u.groups);
    const int pos = a.positions[tok];
    Pieces<T> nx;
    Pieces<G> ng;
    auto load = [&](int gr) __attribute__((always_inline)) {
      const int h = gr * HPG + lane / LPR, hk = h - a.Hq;
      const bool isq = h < a.Hq;
      if (h >= heads) return;
      const G* gp = isq ? (const G*)a.dq_out + ((size_t)tok * a.Hq + h) * D
                        : (const G*)a.dk_out + ((size_t)tok * a.Hkv + hk) * D;
      ng.load(gp + t.e0, gp + t.e1);
      const T* row = isq ? (const T*)a.q + tok * a.q_stride + h * D : (const T*)a.k + tok * a.k_stride + hk * D;
      if (isq ? a.wq != nullptr : a.wk != nullptr) nx.load(row + t.e0, row + t.e1);
    };
    load(g0);
    t.at(pos, a.rot_scale);
    for (int gr = g0; gr < g1; ++gr) {
      const int h = gr * HPG + lane / LPR;
      const bool live = h < heads, isq = h < a.Hq;
      const int hk = h - a.Hq;
      const bool norm = isq ? a.wq != nullptr : a.wk != nullptr;
      float x[8], g[8];
      nx.get(x);
      ng.get(g);
      if (gr + 1 < g1) load(gr + 1);
      t.template apply<true>(g);
      float ss = 0.0f, dot = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
      ss = row_sum<LPR>(ss);
      const float rs = norm ? 1.0f / sqrtf(ss * (1.0f / D) + a.eps) : 1.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= rs;
        const float dw = g[i] * x[i];
        sq[i] += live && isq ? dw : 0.0f;
        sk[i] += live && !isq ? dw : 0.0f;
        g[i] *= isq ? wq[i] : wk[i];
        dot += g[i] * x[i];
      }
      dot = row_sum<LPR>(dot) * (1.0f / D);
      if (!live) continue;
      if (norm) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = rs * (g[i] - x[i] * dot);
      }
      O* o = isq ? (O*)a.dq + tok * a.q_out_stride + h * D : (O*)a.dk + tok * a.k_out_stride + hk * D;
      store_pieces(o + t.e0, o + t.e1, g);
    }
  }
  if (!a.ws) return;  // no norm: no weights
  __shared__ float part[kRopeWaves * HPG][2][D];
  const int row = wave * HPG + lane / LPR;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = i < 4 ? t.e0 + i : t.e1 + i - 4;
    part[row][0][e] = sq[i];
    part[row][1][e] = sk[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * D; c += kWave * kRopeWaves) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < kRopeWaves * HPG; ++j) s += (&part[j][0][0])[c];
    a.ws[(size_t)blockIdx.x * 2 * D + c] = s;
  }
}

// dwq and dwk from the partial rows: a workgroup per 16 columns, 64 rows at a
// time with the loads of eight rounds in flight, then the 64 sums of a column
// in order.  (16 rows at a time, a load after the other: 18 us for 1024 rows.)
constexpr int kDwRows = 64;
__global__ __launch_bounds__(16 * kDwRows) void hyb_rope_dw_kernel(const float* ws, int rows, int d, float* dwq, float* dwk) {
  __shared__ float part[kDwRows][17];
  const int c = threadIdx.x & 15, j = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float s = 0.0f;
#pragma unroll 8
  for (int i = j; i < rows; i += kDwRows) s += ws[(size_t)i * 2 * d + col];
  part[j][c] = s;
  __syncthreads();
  if (j != 0) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < kDwRows; ++i) s += part[i][c];
  float* o = col < d ? dwq : dwk;
  if (o) o[col % d] = s;
}

// Workgroups at most.  The forward's waves take one unit each, so that the rows on
// their way at a time are neighbours in memory (65536 tokens of 16 and 4 heads, d = 128,
// on one card: by 2048 workgroups in rounds 1.16 times as long, with the next unit's loads
// ahead of the last stores 1.31 times; with stores that bypass the caches 0.93 times, which
// the attention that reads the rows next pays back).  The gradient's leave a partial row each, which the
// weights' kernel reads (16384 tokens 49 us with 1024, 55 with 512, 51 with 2048).
constexpr int kRopeGrid = 1 << 20;
constexpr int kRopeBackwardGrid = 1024;

static int rope_backward_rows(const RopeArgs& a, RopeUnits* u) {
  *u = rope_units(a.N, a.Hq + a.Hkv, 512 / a.D, 256 * 8);
  return (int)std::min<long>((u->n + kRopeWaves - 1) / kRopeWaves, kRopeBackwardGrid);
}

size_t rope_backward_ws_bytes(const RopeArgs& a) {
  if (a.N == 0) return 0;
  RopeUnits u;
  return (size_t)rope_backward_rows(a, &u) * 2 * a.D * sizeof(float);
}

template <typename T, typename O, int D, bool INTER>
static void rope_go(const RopeArgs& a, hipStream_t st) {
  const RopeUnits u = rope_units(a.N, a.Hq + (a.slots ? 2 : 1) * a.Hkv, 512 / D, 256 * 16);
  const dim3 grid((unsigned)std::min<long>((u.n + kRopeWaves - 1) / kRopeWaves, kRopeGrid));
  if (a.slots)
    hipLaunchKernelGGL((hyb_rope_kernel<T, O, D, INTER, true>), grid, dim3(kWave * kRopeWaves), 0, st, a, u);
  else
    hipLaunchKernelGGL((hyb_rope_kernel<T, O, D, INTER, false>), grid, dim3(kWave * kRopeWaves), 0, st, a, u);
}

template <typename T, typename G, typename O, int D, bool INTER>
static void rope_backward_go(const RopeArgs& a, hipStream_t st) {
  RopeUnits u;
  const int rows = rope_backward_rows(a, &u);
  hipLaunchKernelGGL((hyb_rope_backward_kernel<T, G, O, D, INTER>), dim3(rows), dim3(kWave * kRopeWaves), 0, st, a, u);
}

template <typename F>
static void rope_shape(const RopeArgs& a, F&& f) {
  const auto yes = std::true_type{};
  const auto no = std::false_type{};
  if (a.D == 64)
    a.interleaved ? f(std::integral_constant<int, 64>{}, yes) : f(std::integral_constant<int, 64>{}, no);
  else
    a.interleaved ? f(std::integral_constant<int, 128>{}, yes) : f(std::integral_constant<int, 128>{}, no);
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t st) {
  auto go = [&](auto t, auto o) {
    typedef decltype(t) T;
    typedef decltype(o) O;
    rope_shape(a, [&](auto d, auto inter) { rope_go<T, O, decltype(d)::value, decltype(inter)::value>(a, st); });
  };
  if (a.dtype == 1)
    a.out_f32 ? go(bf16{}, float{}) : go(bf16{}, bf16{});
  else
    go(float{}, float{});
  return hipGetLastError();
}

hipError_t launch_rope_backward(const RopeArgs& a, hipStream_t st) {
  auto go = [&](auto t, auto g, auto o) {
    typedef decltype(t) T;
    typedef decltype(g) G;
    typedef decltype(o) O;
    rope_shape(a, [&](auto d, auto inter) {
      rope_backward_go<T, G, O, decltype(d)::value, decltype(inter)::value>(a, st);
    });
  };
  if (a.N == 0) {
    // (the weights' gradient is a sum over no rows)
  } else if (a.dtype == 1) {
    if (a.grad_dtype == 1)
      a.out_f32 ? go(bf16{}, bf16{}, float{}) : go(bf16{}, bf16{}, bf16{});
    else
      a.out_f32 ? go(bf16{}, float{}, float{}) : go(bf16{}, float{}, bf16{});
  } else {
    a.grad_dtype == 1 ? go(float{}, bf16{}, float{}) : go(float{}, float{}, float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.dwq && !a.dwk)) return e;
  RopeUnits u;
  const int rows = a.N > 0 ? rope_backward_rows(a, &u) : 0;
  hipLaunchKernelGGL(hyb_rope_dw_kernel, dim3(2 * a.D / 16), dim3(16 * kDwRows), 0, st, a.ws, rows, a.D, a.dwq, a.dwk);
  return hipGetLastError();
}

}  // namespace hyb
