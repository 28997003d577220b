// softmax_q8.hip -- softmax attention of the active block over a paged KV cache in 8
// bits (e4m3 codes, a power-of-two scale per block of tokens and KV head) and the block
// itself, over the whole prefix or its window and first tokens.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(q_i k_j / sqrt(d)),
//   k_j = 2^ek c_j, v_j = 2^ev c'_j for the codes c, c' of cached tokens,
//   over the cached tokens seen and the block's (unquantised) own
//
// The keys are cut into ranges and the ranges' results merged as over an unquantised
// cache (softmax_prefix.h); a tile is 32 cached tokens, which share a page and a scale,
// and the block is the last tile.
//
// Bound: memory where a KV head's queries fit one tile of 32 columns (a token of 1 byte per entry is read
// once for 4 heads' products of 4 d operations), the matrix cores and the conversions of the codes beside
// them where they fill four.  Two kernels: one whose waves convert codes as they become operands, for 32
// columns, and one that converts a tile once for 128, chosen by time (q8_way).
//
// Measured, bf16, 16 and 4 heads of d = 128, calls one after the other: one token of 64 requests of 16384
// tokens 173 us (6.2 TB/s), of one of 32768 19 us; 32 blocks of 32 over 32768 tokens 349 to 365 us (770
// TFLOP/s); 24 blocks of every length over a window of 1024 25 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fp8.h"
#include "launch_cache.h"
#include "softmax_prefix.h"

namespace hyb {

// A tile of 32 rows of D codes in LDS, put there by 16-byte copies: chunk c of K's row t
// sits at c ^ kswz(t), so that the 16 rows which fill the banks have 16 places for
// one chunk, and of V's at c ^ vswz(t), so that the rows r .. r + 3 and r + 8 .. r + 11 of
// two neighbouring chunks, which a transposing read takes, fall in distinct banks.
template <int D>
struct Q8Tile {
  static constexpr int CPR = D / 16;           // chunks per row
  static constexpr int RPI = kWave / CPR;      // rows per copy instruction
  static constexpr int IK = kTile / RPI;       // copies per tile
  static constexpr int kBytes = kTile * D;
  __device__ static constexpr int kswz(int t) { return D == 128 ? (t >> 1) & 7 : (t >> 2) & 3; }
  __device__ static constexpr int vswz(int t) {
    return D == 128 ? 2 * ((t >> 1) & 1) + 4 * ((t >> 3) & 1) : 2 * ((t >> 3) & 1);
  }
  int krow, kx, vrow, vx;  // this lane's row operand, and its transposing read
  __device__ inline explicit Q8Tile(int lane) {
    const int li = lane & 31, hh = lane >> 5, i = lane & 15, b = (lane >> 4) & 1;
    krow = li * D;
    kx = 16 * (hh ^ kswz(li));
    // lane pair i / 2 addresses row 4 hh + (0 .. 3, 8 .. 11)[i / 2], 16 columns of it
    const int r = 4 * hh + (i / 2 & 3) + 8 * (i / 8);
    vrow = r * D + 8 * (i & 1);
    vx = 16 * (b ^ vswz(r));
  }
  // codes 32 i + 16 hh .. + 15 of row li
  __device__ inline uint4 row(const uint8_t* t, int i) const {
    return *reinterpret_cast<const uint4*>(t + krow + (kx ^ (32 * i)));
  }
  // column 32 ct + li at the rows row_of(8 ks + e, hh), e = 0 .. 7.  In each 16-lane
  // quarter the read gives lane i byte i % 8 of the 8-byte pieces addressed by
  // lanes i / 8 + 2 e.
  __device__ inline uint2 column(const uint8_t* t, int ct, int ks) const {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (__attribute__((address_space(3))) i32x2*)(t + 16 * ks * D + vrow + (vx ^ (32 * ct))));
    return uint2{(uint32_t)x[0], (uint32_t)x[1]};
  }
};

// As buf_to_lds16, past the caches: for what no one else reads.
__device__ inline void buf_to_lds16_once(__amdgpu_buffer_rsrc_t r, void* lds, int voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, voff, 0, 0, 2);
}

// A range's tiles: where they are and how a wave copies one.
template <int D>
struct Q8Tiles {
  typedef Q8Tile<D> QT;
  const uint8_t *kc, *vc;  // pools at the KV head
  SpSeen seen;
  int t0, nt, P, page_shift, p0, pa, pskip;
  int stride;  // codes from a token to the next
  const int* pages;

  // All threads of the workgroup; ends with a barrier.  `lds` holds kMaxRangePages numbers.
  __device__ inline Q8Tiles(const SoftmaxQ8Args& a, const SpRange& rg, int g, int P_, int* lds) {
    kc = (const uint8_t*)a.k_cache + g * D;
    vc = (const uint8_t*)a.v_cache + g * D;
    seen = sp_seen<2>(a, rg.b);
    t0 = rg.t0, nt = rg.nt, P = P_;
    page_shift = a.page_shift;
    stride = a.s.Hkv * D;
    pages = lds;
    // the range's pages (page index p0 + e at e; behind page pa, the last before the
    // skipped tiles, p0 + e + pskip), clamped to the pool
    p0 = rg.lo >> page_shift;
    pa = 0x7fffffff;
    pskip = 0;
    if (seen.skip > 0 && t0 < seen.st && t0 + nt > seen.st) {
      pa = (seen.st * kTile - 1) >> page_shift;
      pskip = max(0, ((seen.st + seen.skip) * kTile >> page_shift) - pa - 1);
    }
    const int32_t* ptab = a.page_table + (size_t)rg.b * a.max_pages;
    const int chi = min(rg.hi, P);
    const int np = chi > rg.lo ? ((chi - 1) >> page_shift) - p0 + 1 - pskip : 0;
    for (int e = threadIdx.x; e < np; e += blockDim.x)
      lds[e] = sp_page(a, ptab, (p0 + e + (p0 + e > pa ? pskip : 0)) << page_shift);
    __syncthreads();
  }
  __device__ inline int first_key(int i) const { return seen.tile(t0 + i) * kTile; }
  // Page of the tile at j0 (cached).
  __device__ inline int page(int j0) const {
    const int pi = j0 >> page_shift;
    return pages[pi - p0 - (pi > pa ? pskip : 0)];
  }
  // Bytes of the K and V scales of the tile at j0: K's low.
  __device__ inline int scales(const SoftmaxQ8Args& a, int g, int j0) const {
    const size_t row = ((size_t)page(j0) << page_shift) + (j0 & ((1 << page_shift) - 1));
    const size_t at = (row >> a.sb_shift) * a.s.Hkv + g;
    return a.k_scales[at] | a.v_scales[at] << 8;
  }
  // Whether keys j0 .. j0 + 31 are all cached and seen.
  __device__ inline bool whole(int j0) const { return j0 + kTile <= P && !seen.cuts(j0); }
  __device__ inline bool sees(int j) const { return j < P && !seen.hides(j); }
  // Row t of the tile at j0, or, where that is not seen, one of the tile that is: its
  // weight is zero, and what the row holds may be anything.
  __device__ inline int row(int j0, int t, bool all) const {
    if (all) return t;  // uniform
    int j = min(j0 + t, P - 1);
    if (seen.hides(j)) j = seen.he < min(j0 + kTile, P) ? seen.he : seen.hs - 1;
    return j - j0;
  }
  // K (kv = 0) or V of the tile at j0 into dst; 16 bytes per lane and copy.
  template <bool ONCE>
  __device__ inline void copy(int kv, int j0, uint8_t* dst, int lane) const {
    const size_t row0 = ((size_t)__builtin_amdgcn_readfirstlane(page(j0)) << page_shift) + (j0 & ((1 << page_shift) - 1));
    const uint8_t* base = (kv == 0 ? kc : vc) + row0 * stride;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, kTile * stride, kBufferWord3);
    const bool all = whole(j0);  // uniform
#pragma unroll
    for (int u = 0; u < QT::IK; ++u) {
      const int t = u * QT::RPI + lane / QT::CPR;
      const int c = lane % QT::CPR ^ (kv == 0 ? QT::kswz(t) : QT::vswz(t));
      const int at = row(j0, t, all) * stride + c * 16;
      if constexpr (ONCE)
        buf_to_lds16_once(rs, dst + u * QT::RPI * D, at);
      else
        buf_to_lds16(rs, dst + u * QT::RPI * D, at, 0);
    }
  }
};

// What a wave keeps of its 32 columns: the weights' reference in the log2 domain
// (finite, so that a wave without tiles weighs nothing; it moves only when a
// maximum passes it by 2^8), their sum over the lane's rows, and the weighted sums of V^T.
template <typename T, int D>
struct Q8Acc {
  typedef Mma<T> M;
  typedef typename M::op_t op_t;
  static constexpr int KD = D / M::KW, KL = kTile / M::KW, NCT = D / kTile;
  // Entry of a row that lane half hh contracts at step ks, element e: any order will do
  // that both operands share, and here 16 codes of a row are one read.
  static constexpr int SPR = 16 / M::E;  // steps of a read
  __device__ static constexpr int entry(int ks, int hh) { return ks / SPR * 32 + 16 * hh + ks % SPR * M::E; }
  float m = -1e30f, l = 0.0f;
  f32x16 acc[NCT];
  __device__ inline Q8Acc() {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  }
  // Scores (K Q^T) of a tile of codes, without their scale.
  __device__ static inline f32x16 scores(const Q8Tile<D>& qt, const uint8_t* kt, const op_t (&qop)[KD]) {
    f32x16 sc = {};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 x = qt.row(kt, i);
      if constexpr (sizeof(T) == 2) {
        sc = M::mma(fp8_bf16(x.x, x.y, 1.0f), qop[2 * i], sc);
        sc = M::mma(fp8_bf16(x.z, x.w, 1.0f), qop[2 * i + 1], sc);
      } else {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const f32x4 k = fp8_f32(w[y], 1.0f);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = M::mma(k[e], qop[16 * i + 4 * y + e], sc);
        }
      }
    }
    return sc;
  }
  // Weights of a tile's masked scores (in p), for a scale into the log2 domain.
  __device__ inline void weights(const f32x16& sc, float scale, float (&p)[16]) {
    float mt = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
    mt = fmaxf(mt, xor32(mt)) * scale;
    if (__any(mt > m + 8.0f)) {
      mma_settle<T>();
      const float mn = mt > m + 8.0f ? mt : m;
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[ct][e] *= corr;
      m = mn;
    }
    float sum[4] = {};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -m));
      sum[e % 4] += p[e];
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // A tile of cached tokens at j0 with its scales' bytes.
  __device__ inline void add(const Q8Tiles<D>& t, const Q8Tile<D>& qt, int j0, const uint8_t* kt, const uint8_t* vt,
                             int bytes, const op_t (&qop)[KD], float scale, int hh) {
    f32x16 sc = scores(qt, kt, qop);
    mma_settle<T>();
    if (!t.whole(j0)) {  // uniform
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = t.sees(j0 + row_of(e, hh)) ? sc[e] : -INFINITY;
    }
    const float fk = scale * scale_of(bytes & 255), fv = scale_of(bytes >> 8);
    float p[16];
    weights(sc, fk, p);
    if constexpr (sizeof(T) == 2) {
      // The weights enter P V rounded to bf16 (each off by at most 2^-8 of itself;
      // products of fp32 run at 1/16 of the rate); their sum is over the unrounded ones.
      op_t pop[KL];
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) pop[ks] = cvt_op<bf16>(&p[ks * 8]);
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int ks = 0; ks < KL; ++ks) {
          const uint2 x = qt.column(vt, ct, ks);
          acc[ct] = M::mma(fp8_bf16(x.x, x.y, fv), pop[ks], acc[ct]);
        }
    } else {
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const uint2 x = qt.column(vt, ct, ks);
          const f32x4 lo = fp8_f32(x.x, fv), hi = fp8_f32(x.y, fv);
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[ct] = M::mma(e < 4 ? lo[e] : hi[e - 4], p[8 * ks + e], acc[ct]);
        }
    }
  }
  // The block's tile: n rows of T in LDS, D entries each and 16 bytes apart from the next.
  static constexpr int LD = D + 16 / (int)sizeof(T);
  __device__ inline void add_block(const T* kb, const T* vb, int n, const op_t (&qop)[KD], float scale, int li, int hh) {
    f32x16 sc = {};
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) sc = M::mma(load_op<T>(kb + li * LD + entry(ks, hh)), qop[ks], sc);
    mma_settle<T>();
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = row_of(e, hh) < n ? sc[e] : -INFINITY;
    float p[16];
    weights(sc, scale, p);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks)
        acc[ct] = M::mma(load_rows_op<T>(vb + ct * kTile + li, LD, ks, hh, kTile, false), cvt_op<T>(&p[ks * M::E]), acc[ct]);
  }
};

// Where the L queries of a KV head's query heads are, one head after the other, in
// tiles of 32 columns: `groups` of them.
__host__ __device__ inline int q8_groups(const Shape& s) { return (s.Hq / s.Hkv * s.L + kTile - 1) / kTile; }

// A workgroup answers 32 columns over a range of keys: its waves take the
// range's tiles in turn, each through copies of its own (R slots, no barrier in the loop)
// and sums of its own, joined in LDS at the end.  The codes are converted as they become
// operands.  Eight waves: a tile is one chain of reads, conversions, products and weights, which
// two waves per SIMD overlap (a tile of 32 columns at d = 128 takes a CU 0.32 us with four waves
// of four slots, 0.18 so; 64 requests of 16384 tokens 214 and 194 us).  fp32 at d = 128 has
// room for four.
template <typename T, int D>
__host__ __device__ constexpr int q8_token_threads() {
  return kWave * (sizeof(T) == 4 && D == 128 ? 4 : 8);
}
template <typename T, int D, bool ONCE>
__global__ __launch_bounds__((q8_token_threads<T, D>())) void hyb_q8_token_kernel(SoftmaxQ8Args a, SpCut cut) {
  typedef Q8Acc<T, D> A;
  typedef Q8Tile<D> QT;
  constexpr int NCT = A::NCT, NW = q8_token_threads<T, D>() / kWave, R = 2;
  struct alignas(16) Slot {
    uint8_t k[QT::kBytes], v[QT::kBytes];
  };
  struct Block {
    T k[kTile * A::LD], v[kTile * A::LD];
  };
  union Smem {
    struct {
      Slot ring[NW][R];
    } loop;
    f32x4 parts[NW][NCT * 4][kWave];
    __device__ Smem() {}
  };
  __shared__ alignas(16) Smem sh;
  __shared__ alignas(16) Block blk;
  __shared__ float refs[NW][kTile], sums[NW][kTile];
  __shared__ int pages[kMaxRangePages];
  __shared__ uint16_t bytes[kMaxRange / kTile + 2];

  const int lane = threadIdx.x & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L, G = Hq / Hkv;
  int at, hg;
  sp_place(q8_groups(a.s), at, hg);
  const int g = at % Hkv, r = at / Hkv;
  const SpRange rg = sp_range<2>(a, sp_even_plan(a, cut), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int Lb = sp_block<2>(a, rg.b), P = min(max(a.prefix_len[rg.b], 0), a.max_prefix);
  // this lane's column: query i of head h
  const int col = hg * kTile + li, hl = col / L, i = col - hl * L, h = g * G + hl;
  const bool mine = hl < G && i < Lb;
  typename A::op_t qop[A::KD];
  {
    const T* row = (const T*)a.q + (((size_t)rg.b * L + (mine ? i : 0)) * Hq + (mine ? h : g * G)) * D;
#pragma unroll
    for (int ks = 0; ks < A::KD; ++ks) qop[ks] = keep_if<T>(mine, load_op<T>(row + A::entry(ks, hh)));
  }
  const Q8Tiles<D> t(a, rg, g, P, pages);
  const QT qt(lane);
  const bool block = rg.hi > (P + kTile - 1) / kTile * kTile;  // the range's last tile is the block's
  const int nt = rg.nt - (block ? 1 : 0), my = (nt - w + NW - 1) / NW;  // cached tiles, this wave's
  auto issue = [&](int n, Slot& s) __attribute__((always_inline)) {
    if (n >= my) return;
    const int j0 = t.first_key(w + NW * n);
    t.template copy<ONCE>(0, j0, s.k, lane);
    t.template copy<ONCE>(1, j0, s.v, lane);
  };
  // The first tile beside the scales and the block (its page is there since the barrier at the end
  // of t's making): one token over 32768 19.4 us after them, 18.7 so.  Not where the cache goes
  // past the chip's caches: 64 requests of 16384 tokens 172 and 177.
  if constexpr (!ONCE) issue(0, sh.loop.ring[w][0]);
  for (int e = threadIdx.x; e < nt; e += NW * kWave) bytes[e] = (uint16_t)t.scales(a, g, t.first_key(e));
  if (block) {  // rows past the block's are the last again
    constexpr int EPC = 16 / (int)sizeof(T), CPR = D / EPC;
    const size_t row0 = (size_t)rg.b * L;
    for (int x = threadIdx.x; x < kTile * CPR; x += NW * kWave) {
      const size_t src = ((row0 + min(x / CPR, Lb - 1)) * Hkv + g) * D + x % CPR * EPC;
      const int dst = x / CPR * A::LD + x % CPR * EPC;
      *reinterpret_cast<uint4*>(&blk.k[dst]) = *reinterpret_cast<const uint4*>((const T*)a.k + src);
      *reinterpret_cast<uint4*>(&blk.v[dst]) = *reinterpret_cast<const uint4*>((const T*)a.v + src);
    }
  }
  __syncthreads();
  if constexpr (ONCE) issue(0, sh.loop.ring[w][0]);
  const float scale = kLog2e / sqrtf((float)D);
  A acc;
  auto step = [&](int n, auto S) __attribute__((always_inline)) {
    constexpr int SV = decltype(S)::value;
    if (n >= my) return;
    issue(n + 1, sh.loop.ring[w][(SV + 1) % R]);
    if (n + 1 < my) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * QT::IK) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const Slot& s = sh.loop.ring[w][SV];
    acc.add(t, qt, t.first_key(w + NW * n), s.k, s.v, bytes[w + NW * n], qop, scale, hh);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read
  };
  for (int n = 0; n < my; n += R) {
    step(n, std::integral_constant<int, 0>{});
    step(n + 1, std::integral_constant<int, 1>{});
  }
  if (block && w == nt % NW) acc.add_block(blk.k, blk.v, Lb, qop, scale, li, hh);

  // The waves' sums over one reference: a wave scales its own and leaves them in LDS,
  // then joins its share of every column's entries.
  mma_settle<T>();
  const float l = acc.l + xor32(acc.l);
  if (hh == 0) refs[w][li] = acc.m;
  lds_barrier();  // (and the slots are free)
  float mm = refs[0][li];
#pragma unroll
  for (int x = 1; x < NW; ++x) mm = fmaxf(mm, refs[x][li]);
  const float f = __builtin_amdgcn_exp2f(acc.m - mm);
  if (hh == 0) sums[w][li] = l * f;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x16& y = acc.acc[ct];
      sh.parts[w][ct * 4 + e][lane] = f32x4{y[4 * e] * f, y[4 * e + 1] * f, y[4 * e + 2] * f, y[4 * e + 3] * f};
    }
  lds_barrier();
  if (!mine) return;
  float den = 0.0f;
#pragma unroll
  for (int x = 0; x < NW; ++x) den += sums[x][li];
  constexpr int PW = NCT * 4 / NW;  // pieces of four entries per wave
  static_assert(PW * NW == NCT * 4, "every piece has its wave");
#pragma unroll
  for (int y = w * PW; y < w * PW + PW; ++y) {
    f32x4 o = {};
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const f32x4 z = sh.parts[x][y][lane];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += z[k];
    }
    sp_put<T, D>(a, rg, r, h, i, y / 4 * kTile + row_of(y % 4 * 4, hh), o, den);
  }
  if (w == 0 && hh == 0) sp_put_sum<D>(a, rg, r, h, i, mm, den);
}

// Blocks (bf16; more than 32 columns): a wave answers 32 columns, and the four waves of a
// half share its tiles; with H = 2 the two halves of a workgroup take the range's tiles in turn
// and join their sums in LDS, with H = 1, where workgroups are many, two of them share a CU.
// A tile's codes go through registers, A tiles ahead, and into LDS as bf16 values, scales
// included, so that each is converted once for four tiles of columns; the tiles are then read as
// those of a bf16 cache.  Step n forms the scores of tile n + 1 while it takes the weights of
// tile n (two independent chains, whose MFMAs and VALU instructions interleave), and puts tile
// n + 2 into the slot of tile n - 1.
template <int D, int H>
__global__ __launch_bounds__(kWave * 4 * H, 2) void hyb_q8_block_kernel(SoftmaxQ8Args a, SpCut cut) {
  typedef Mma<bf16> M;
  typedef M::op_t op_t;
  typedef RowColTile<D> RT;
  constexpr int KD = D / M::KW, KL = kTile / M::KW, NCT = D / kTile, NW = 4, R = 3, A = 3;
  constexpr int CPR = D / 16, PK = kTile * CPR;          // 16-code pieces of a row, of a tile of K or V
  constexpr int PT = 2 * PK / (kWave * NW);              // pieces of a thread of the half and tile
  static_assert(PT >= 1 && PK % kWave == 0, "a wave's pieces are all of K or of V");
  struct alignas(16) Slot {
    bf16 x[2][kTile * D];
  };
  constexpr int NH = NCT / 2;  // groups of 32 entries that a half joins
  union Smem {
    Slot ring[H][R];
    f32x4 parts[H][NW][NH * 4][kWave];  // [for half]
    __device__ Smem() {}
  };
  __shared__ alignas(16) Smem sh;
  __shared__ float refs[H][NW][kTile], sums[H][NW][kTile];
  __shared__ int pages[kMaxRangePages];
  // Of the range's cached tiles, and of one more, hidden whole, behind them: the offset of
  // their first row in the pools (kPartial in the high word: not all of its rows are seen),
  // and the bytes of their scales.
  constexpr uint32_t kPartial = 1u << 31;
  __shared__ uint2 places[kMaxRange / kTile + 3];
  __shared__ uint16_t bytes[kMaxRange / kTile + 3];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = wave / NW, w = wave % NW;
  Slot(&ring)[R] = sh.ring[half];
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L, G = Hq / Hkv;
  int at, hg;
  sp_place((q8_groups(a.s) + NW - 1) / NW, at, hg);
  const int g = at % Hkv, r = at / Hkv;
  const SpRange rg = sp_range<2>(a, sp_even_plan(a, cut), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int Lb = sp_block<2>(a, rg.b), P = min(max(a.prefix_len[rg.b], 0), a.max_prefix);
  const int col = (hg * NW + w) * kTile + li, hl = col / L, i = col - hl * L, h = g * G + hl;
  const bool mine = hl < G && i < Lb;
  op_t qop[KD];
  {
    const bf16* row = (const bf16*)a.q + (((size_t)rg.b * L + (mine ? i : 0)) * Hq + (mine ? h : g * G)) * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) qop[ks] = keep_if<bf16>(mine, load_op<bf16>(row + ks * M::KW));
  }
  const Q8Tiles<D> t(a, rg, g, P, pages);
  const RT rt(lane);
  // The list: the block's tile first, if it is the range's, then the cached ones, nc of
  // them; this half's tile n is the list's H n + half.  The halves have the same number:
  // one that is past the list's end takes the hidden one.
  const int nb = rg.hi > (P + kTile - 1) / kTile * kTile ? 1 : 0, nc = rg.nt - nb, ntiles = (rg.nt + H - 1) / H;
  const bool first_is_block = half < nb;
  for (int e = threadIdx.x; e <= nc; e += blockDim.x) {
    const int j0 = t.first_key(max(0, min(e, nc - 1)));
    const size_t row = ((size_t)t.page(j0) << t.page_shift) + (j0 & ((1 << t.page_shift) - 1));
    const size_t off = nc > 0 ? row * t.stride : 0;
    places[e] = uint2{(uint32_t)off, (uint32_t)(off >> 32) | (e == nc || !t.whole(j0) ? kPartial : 0u)};
  }
  auto entry = [&](int n) __attribute__((always_inline)) { return max(0, min(H * n + half - nb, nc)); };
  lds_barrier();  // (the places are there)

  // 16-code piece y of a tile: a write puts down eight lanes' 16 bytes at once, so four pieces of
  // a row go with four of the row four on, whose swizzle differs in the lowest bit: one's even
  // chunks and the other's fall in distinct banks.
  auto piece = [&](int y, int& row, int& c16) __attribute__((always_inline)) {
    c16 = (y & 3) | (D == 128 ? y >> 1 & 4 : 0);
    const int x = D == 128 ? y >> 4 : y >> 3;
    row = (y & 4) | (x & 3) | (x >> 2) << 3;
  };
  uint4 next[A][PT];  // codes of tiles on their way
  int voff[PT], dst0[PT], dst1[PT];  // this thread's pieces: their offsets in a tile in the pools, and in a slot
  const int kvs = PT > 1 ? 0 : w * kWave / PK;
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    int row, c16;
    piece((u * kWave * NW + w * kWave + lane) % PK, row, c16);
    voff[u] = row * t.stride + c16 * 16;
    dst0[u] = row * D + ((2 * c16) ^ RT::swz(row)) * 8;
    dst1[u] = row * D + ((2 * c16 + 1) ^ RT::swz(row)) * 8;
  }
  auto kind = [&](int u) __attribute__((always_inline)) { return PT > 1 ? u * kWave * NW / PK : kvs; };  // K's or V's
  // Always as many loads, whatever n is: where some were left out, the compiler, which
  // counts what is in flight, would wait for all of them.  (Without cached tiles the buffer is
  // empty, and nothing is loaded.)
  const int span = nc > 0 ? kTile * t.stride : 0;
  auto fetch = [&](int n, uint2 place, uint4 (&c)[PT]) __attribute__((always_inline)) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(place.x), hi = __builtin_amdgcn_readfirstlane(place.y);
    const size_t off = (size_t)(hi & ~kPartial) << 32 | lo;
    int at[PT];
#pragma unroll
    for (int u = 0; u < PT; ++u) at[u] = voff[u];
    if (hi & kPartial) {  // uniform; (any row will do for the hidden tile)
      const int j0 = t.first_key(max(0, min(entry(n), nc - 1)));
#pragma unroll
      for (int u = 0; u < PT; ++u) {
        int row, c16;
        piece((u * kWave * NW + w * kWave + lane) % PK, row, c16);
        at[u] = t.row(j0, row, t.whole(j0)) * t.stride + c16 * 16;
      }
    }
#pragma unroll
    for (int u = 0; u < PT; ++u) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>((kind(u) == 0 ? t.kc : t.vc) + off), 0, span, kBufferWord3);
      c[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, at[u], 0, 0));
    }
  };
  auto put = [&](int by, const uint4 (&c)[PT], Slot& s) __attribute__((always_inline)) {
    const int two = __builtin_amdgcn_readfirstlane(by);
#pragma unroll
    for (int u = 0; u < PT; ++u) {
      const float f = scale_of(kind(u) == 0 ? two & 255 : two >> 8);
      *reinterpret_cast<bf16x8*>(s.x[kind(u)] + dst0[u]) = fp8_bf16(c[u].x, c[u].y, f);
      *reinterpret_cast<bf16x8*>(s.x[kind(u)] + dst1[u]) = fp8_bf16(c[u].z, c[u].w, f);
    }
  };
  // The block's rows as they are; those past its last are the last again.
  auto put_block = [&](Slot& s) __attribute__((always_inline)) {
    for (int x = w * kWave + lane; x < 2 * kTile * D / 8; x += kWave * NW) {
      const int kv = x / (kTile * D / 8), row = x / (D / 8) % kTile, c8 = x % (D / 8);
      const bf16* src = (const bf16*)(kv == 0 ? a.k : a.v) + (((size_t)rg.b * L + min(row, Lb - 1)) * Hkv + g) * D + c8 * 8;
      *reinterpret_cast<bf16x8*>(&s.x[kv][row * D + (c8 ^ RT::swz(row)) * 8]) = load_op<bf16>(src);
    }
  };

  const float scale = kLog2e / sqrtf((float)D);
  float m = -1e30f, l = 0.0f;
  f32x16 acc[NCT], sc;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  auto scores = [&](const Slot& s) __attribute__((always_inline)) {
    f32x16 x = {};
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) x = M::mma(rt.row_op(s.x[0], ks), qop[ks], x);
    return x;
  };
  // Takes the scores of tile n: masks, maximum, reference (which moves only when a
  // maximum passes it by 2^8).
  auto take = [&](int n, const f32x16& s, bool partial) __attribute__((always_inline)) {
    sc = s;
    if (partial) {  // uniform
      const bool block = n == 0 && first_is_block, past = !block && entry(n) == nc;
      const int j0 = block || past ? 0 : t.first_key(entry(n));
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = j0 + row_of(e, hh);
        sc[e] = !past && (block ? j < Lb : t.sees(j)) ? sc[e] : -INFINITY;
      }
    }
    float mt = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
    mt = fmaxf(mt, xor32(mt)) * scale;
    if (__any(mt > m + 8.0f)) {
      mma_settle<bf16>();
      const float mn = mt > m + 8.0f ? mt : m;
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[ct][e] *= corr;
      m = mn;
    }
  };
  auto compute = [&](auto lastc, int n, const Slot& sn, const Slot& sv, bool partial, auto stage) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(lastc)::value;
    f32x16 x;
    if constexpr (!LAST) x = scores(sn);
    stage();
    float p[16], s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -m));
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      s0 += p[e];
      s1 += p[e + 1];
    }
    l += s0 + s1;
    op_t pop[KL];  // (the weights rounded to bf16 for P V, their sum over the unrounded ones)
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) pop[ks] = cvt_op<bf16>(&p[ks * 8]);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) acc[ct] = M::mma(rt.col_op(sv.x[1], ct, ks), pop[ks], acc[ct]);
    if constexpr (!LAST) take(n + 1, x, partial);
  };
#pragma unroll
  for (int n = 0; n < A; ++n) fetch(n, places[entry(n)], next[n]);
  // (the scales' bytes beside the first tiles)
  for (int e = threadIdx.x; e <= nc; e += blockDim.x)
    bytes[e] = nc > 0 ? (uint16_t)t.scales(a, g, t.first_key(max(0, min(e, nc - 1)))) : 0;
  lds_barrier();  // (the bytes are there)
  if (first_is_block)
    put_block(ring[0]);
  else
    put(bytes[entry(0)], next[0], ring[0]);
  fetch(A, places[entry(A)], next[0]);
  put(bytes[entry(1)], next[1], ring[1]);
  fetch(A + 1, places[entry(A + 1)], next[1]);
  // (what a step takes of a tile as numbers is read a step ahead)
  uint2 place = places[entry(A + 2)];
  int by = bytes[entry(2)];
  uint32_t how = places[entry(1)].y;
  lds_barrier();
  {
    const f32x16 x = scores(ring[0]);
    mma_settle<bf16>();
    take(0, x, first_is_block || (__builtin_amdgcn_readfirstlane(places[entry(0)].y) & kPartial));
  }
  // (R = A: a tile's registers and slot have the same number)
  static_assert(R == A, "one index for both");
  auto step = [&](int n, auto S) __attribute__((always_inline)) {
    constexpr int SV = decltype(S)::value;
    const bool partial = __builtin_amdgcn_readfirstlane(how) & kPartial;
    compute(std::false_type{}, n, ring[(SV + 1) % R], ring[SV], partial, [&]() __attribute__((always_inline)) {
      // every wave has read tile n - 1, whose slot tile n + 2 takes
      put(by, next[(SV + 2) % A], ring[(SV + 2) % R]);
      fetch(n + 2 + A, place, next[(SV + 2) % A]);
      place = places[entry(n + 3 + A)];
      by = bytes[entry(n + 3)];
      how = places[entry(n + 2)].y;
    });
    lds_barrier();
  };
  int n = 0;
  for (; n + R < ntiles; n += R) {
    step(n, std::integral_constant<int, 0>{});
    step(n + 1, std::integral_constant<int, 1>{});
    step(n + 2, std::integral_constant<int, 2>{});
  }
  if (n + 1 < ntiles) step(n, std::integral_constant<int, 0>{});
  if (n + 2 < ntiles) step(n + 1, std::integral_constant<int, 1>{});
  compute(std::true_type{}, ntiles - 1, ring[0], ring[ntiles - 1 - n], false, [] {});
  mma_settle<bf16>();
  l += xor32(l);
  if constexpr (H == 1) {
    if (!mine) return;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sp_put<bf16, D>(a, rg, r, h, i, ct * kTile + row_of(4 * e, hh),
                        f32x4{acc[ct][4 * e], acc[ct][4 * e + 1], acc[ct][4 * e + 2], acc[ct][4 * e + 3]}, l);
    if (hh == 0) sp_put_sum<D>(a, rg, r, h, i, m, l);
  } else {
    // The halves' sums over one reference: each hands over half of the entries and joins
    // the others.
    if (hh == 0) refs[half][w][li] = m;
    lds_barrier();  // (and the slots are free)
    const float mm = fmaxf(refs[0][w][li], refs[1][w][li]), f = __builtin_amdgcn_exp2f(m - mm);
    if (hh == 0) sums[half][w][li] = l * f;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ct / NH != half)
          sh.parts[ct / NH][w][ct % NH * 4 + e][lane] =
              f32x4{acc[ct][4 * e] * f, acc[ct][4 * e + 1] * f, acc[ct][4 * e + 2] * f, acc[ct][4 * e + 3] * f};
    lds_barrier();
    if (!mine) return;
    const float den = sums[0][w][li] + sums[1][w][li];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      if (ct / NH == half)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4 o = sh.parts[half][w][ct % NH * 4 + e][lane];
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] += acc[ct][4 * e + k] * f;
          sp_put<bf16, D>(a, rg, r, h, i, ct * kTile + row_of(4 * e, hh), o, den);
        }
    if (half == 0 && hh == 0) sp_put_sum<D>(a, rg, r, h, i, mm, den);
  }
}

// Merge of few rows' ranges: a workgroup per row, D / 4 threads per range, as many
// ranges at once as it has threads for.  (16 rows of 64 ranges: 27.5 us by eight rows per
// workgroup, one after the other, 4 us so.)
template <typename T, int D>
__global__ __launch_bounds__(256) void hyb_q8_combine_kernel(SoftmaxPrefixArgs a, SpCut cut) {
  constexpr int TPR = D / 4, NG = 256 / TPR;
  __shared__ float most[NG], sums[NG];
  __shared__ f32x4 parts[NG][TPR];
  const SpPlan p = sp_even_plan(a, cut);
  if (p.whole) return;  // every row is already written out
  const int Hq = a.s.Hq, L = a.s.L, lane = threadIdx.x & (kWave - 1);
  const int b = blockIdx.x / (Hq * L), h = blockIdx.x / L % Hq, i = blockIdx.x % L;
  const int n = sp_ranges(p, sp_tiles<2>(a, b));
  if (n <= 1 || i >= sp_block<2>(a, b)) return;  // uniform
  int base = 0;
  for (int b0 = lane; b0 < b; b0 += kWave) base += sp_ranges(p, sp_tiles<2>(a, b0));
  base = wave_all(base, AddOp{});
  const int grp = threadIdx.x / TPR, c = threadIdx.x % TPR;
  const size_t row0 = sp_row(a, base, h, i), step = (size_t)Hq * L;
  const float* wml = sp_ml<D>(a);
  float m = -1e30f, den = 0.0f;
  f32x4 num = {};
#pragma unroll 4
  for (int s = grp; s < n; s += NG) {
    const size_t rr = row0 + s * step;
    const float2 ml = *reinterpret_cast<const float2*>(wml + rr * 2);
    const f32x4 x = *reinterpret_cast<const f32x4*>((const float*)a.ws + rr * D + c * 4);
    const float mn = fmaxf(m, ml.x), f = fast_exp(m - mn), g = fast_exp(ml.x - mn);
    m = mn;
    den = den * f + ml.y * g;
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = num[e] * f + x[e] * g;
  }
  if (c == 0) {
    most[grp] = m;
    sums[grp] = den;
  }
  parts[grp][c] = num;
  __syncthreads();
  if (threadIdx.x >= TPR) return;
  float mm = most[0];
#pragma unroll
  for (int x = 1; x < NG; ++x) mm = fmaxf(mm, most[x]);
  float o[4] = {}, d = 0.0f;
#pragma unroll
  for (int x = 0; x < NG; ++x) {
    const float f = fast_exp(most[x] - mm);
    d += sums[x] * f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += parts[x][c][e] * f;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] /= d;
  store_out4<T>(a.out, (((size_t)b * L + i) * Hq + h) * D + c * 4, o, a.s.out_f32);
}

// Which kernel, its workgroups for a range and KV head, and into how many ranges requests of
// max_seen cached tokens are cut: the least estimated time (us).  The chip takes a
// workgroup per CU at a time; one costs its start and end besides its tiles (at D = 128 0.19 us
// of 32 columns and 0.55 of 128, fp32 1.36, at 64 0.14, 0.4 and 0.62; two of 128 columns without
// halves 1.04, at 64 0.75), and more ranges than one cost a merge and the partial rows.  (The numbers are fitted to 88 shapes of bf16, where what this
// takes is within 0.4% of the best on average.  4 KV heads of 4 query heads, D = 128, blocks of 32,
// the kernel of 32 columns against that of 128 at each one's best ranges: a window of 1024 of 16
// requests 15 and 29 us, of 48 41 and 32; of 4096 of 4 requests 25 and 29, of 24 61 and 57.  Without
// halves against with them: a window of 1024 of 64 requests 38 and 36, of 128 52 and 66.)
struct Q8Way {
  int columns;  // tiles of them per workgroup: 1 or 4
  int halves;
  int wgs, ranges;
};
static Q8Way q8_way(const Shape& s, int max_seen) {
  const int groups = q8_groups(s);
  const double tiles = std::ceil(max_seen / 32.0) + 1, width = s.D == 64 ? 0.72 : 1.0;
  const double rows = (double)s.B * s.Hq * s.L, row = (s.D + 2) / 1e6;  // a partial row's write and read
  Q8Way best = {};
  double least = 0;
  auto take = [&](Q8Way w, double time) {
    if (least == 0 || time < least * 0.98) {
      least = time;
      best = w;
    }
  };
  for (int block = 0; block <= (s.dtype == 1 && groups > 1 ? 1 : 0); ++block) {
    const int per = block ? (groups + 3) / 4 : groups;
    const double wgs = (double)s.B * s.Hkv * per;
    const double tile = s.dtype != 1 ? (s.D == 64 ? 0.62 : 1.36) : (block ? 0.55 : 0.19) * width;
    const double fixed = block ? 11.3 : 8.4;
    // one, and as many as fill the chip once, twice, ..
    for (int rounds = 0; rounds <= 4; ++rounds) {
      const int k = rounds == 0 ? 1 : (int)std::min(256.0 * rounds / wgs, tiles / 4);
      if (k < 1) continue;
      take({block ? 4 : 1, 2, per, k},
           std::ceil(wgs * k / 256) * (std::ceil(tiles / k) * tile + fixed) + (k > 1 ? 6.0 + rows * k * row : 0.0));
    }
    if (block && wgs > 256) take({4, 1, per, 1}, std::ceil(wgs / 512) * (tiles * 1.04 * width + fixed));
  }
  return best;
}
// Ranges per request at most: a plan's ranges are c tiles, an even share of all
// tiles, so that requests of different lengths have one more than that on average.
int softmax_q8_splits(const Shape& s, int max_seen) {
  if (s.B == 0) return 1;
  const int need = (int)(((long)max_seen + s.L + kMaxRange - 1) / kMaxRange);
  const int k = q8_way(s, max_seen).ranges;
  return k == 1 && need <= 1 ? 1 : std::max(k, need) + 1;
}

template <typename T, int D>
static hipError_t q8_go(const SoftmaxQ8Args& a, hipStream_t st) {
  const Q8Way way = q8_way(a.s, a.max_seen);
  SpCut cut = {};
  cut.limit = a.s.B * a.n_split;
  const dim3 grid((unsigned)(a.s.Hkv * way.wgs * cut.limit));
  const dim3 threads((q8_token_threads<T, D>()));
  bool done = false;
  if constexpr (sizeof(T) == 2) {
    // A cache that no second workgroup reads and the chip's caches (256 MB) would not keep until the
    // next call goes past them (64 requests of 16384 tokens, 1 GB, 194 us through them, 173 so;
    // 24 of 8192, 100 MB at D = 64 and read again by the next call, 39 and 42; 16 blocks of 4 tiles of
    // columns, 55 and 63).
    const bool once = way.wgs == 1 && (double)a.s.B * a.s.Hkv * a.max_seen * 2 * D > 256e6;
    done = way.columns == 4 || once;
    if (way.columns == 4 && way.halves == 2)
      hipLaunchKernelGGL((hyb_q8_block_kernel<D, 2>), grid, dim3(kWave * 8), 0, st, a, cut);
    else if (way.columns == 4)
      hipLaunchKernelGGL((hyb_q8_block_kernel<D, 1>), grid, dim3(kWave * 4), 0, st, a, cut);
    else if (once)
      hipLaunchKernelGGL((hyb_q8_token_kernel<T, D, true>), grid, threads, 0, st, a, cut);
  }
  if (!done) hipLaunchKernelGGL((hyb_q8_token_kernel<T, D, false>), grid, threads, 0, st, a, cut);
  if (a.n_split == 1) return hipGetLastError();  // one range: already written out
  const long rows = (long)a.s.B * a.s.Hq * a.s.L, units = (long)a.s.B * a.s.Hq * ((a.s.L + 1024 / D - 1) / (1024 / D));
  if (rows <= 2048 && a.n_split > 4)
    hipLaunchKernelGGL((hyb_q8_combine_kernel<T, D>), dim3((unsigned)rows), dim3(256), 0, st, a, cut);
  else
    hipLaunchKernelGGL((hyb_sp_combine_kernel<T, D, 2>), dim3((unsigned)std::min<long>(units, 2048)), dim3(256), 0, st, a,
                       cut);
  return hipGetLastError();
}

// Threads of the largest launch.
double softmax_q8_threads(const SoftmaxQ8Args& a) {
  const Q8Way way = q8_way(a.s, a.max_seen);
  return 8.0 * kWave * a.s.B * a.n_split * a.s.Hkv * way.wgs;
}

hipError_t launch_softmax_q8(const SoftmaxQ8Args& a, hipStream_t st) {
  if (a.s.dtype == 1) return a.s.D == 64 ? q8_go<bf16, 64>(a, st) : q8_go<bf16, 128>(a, st);
  return a.s.D == 64 ? q8_go<float, 64>(a, st) : q8_go<float, 128>(a, st);
}

}  // namespace hyb
