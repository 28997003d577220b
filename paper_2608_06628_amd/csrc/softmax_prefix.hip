// softmax_prefix.hip -- exact softmax attention of the active block over a
// request's cached prefix plus the block itself: the softmax layer that the
// hybrid layer replaces (Section 2.2 attention without a mask inside the
// block; the comparison of the paper's kernel benchmark, Appendix A).
//
// Split-KV flash decoding.  Keys are indexed in the concatenation
// [k_cache[b][0 .. P_b-1]; k_block[b][0 .. L-1]] and cut into ranges of whole
// 32-key tiles, as many per request as its length asks for (SpPlan).
// One workgroup per (request b, KV head g, range s) with one wave per query
// head of the group (GQA packing: the G heads share every K/V tile through
// LDS).  Each 32-key tile gives Sc^T = K Q^T (keys in rows, one query per
// lane column), an online-softmax update, and O^T += V^T P^T, with P rounded
// once to the operand type and the running sum taken over the rounded
// weights.  A second kernel merges the ranges with their log-sum-exp weights;
// with a single range the first kernel writes the normalised output itself.
//
// The cache is either contiguous per request ([B][max_prefix][Hkv][d]) or
// paged: a pool of fixed-size pages ([n_pages][page][Hkv][d]) and a page table
// per request, as a serving engine's paged KV cache keeps it (Section 3.3).
// The page size is a power of two of at least 32 rows, so a 32-key tile lies
// in one page.  The ring kernel stages its range's page numbers in LDS when
// it starts (a range holds at most kMaxRange keys), so the copies of a tile
// take their page from LDS and no vector load of the page table sits among
// the copies whose counts the ring waits on.
#include <algorithm>
#include <type_traits>

#include "device.h"
#include "launch.h"
#include "softmax_prefix.h"

namespace hyb {

template <typename T, int D, int NG>
struct SpCfg {
  typedef Mma<T> M;
  typedef typename M::op_t op_t;
  static constexpr int KD = D / M::KW;
  static constexpr int KL = kTile / M::KW;
  static constexpr int NCT = D / kTile;
  static constexpr int EPC = 16 / (int)sizeof(T);  // elements per 16 bytes
  static constexpr int KLD = D + EPC;              // K rows: 16-byte pad
  static constexpr int VLD = D + 2 * EPC;          // V rows: 32-byte pad
  static constexpr int CPR = D / EPC;              // 16-byte chunks per row
  static constexpr int NCH = (kTile * CPR + kWave * NG - 1) / (kWave * NG);  // per thread
  struct alignas(16) Smem {
    T k[2][kTile][KLD];
    T v[2][kTile][VLD];
  };
};

constexpr int kMaxGroup = 8;  // query heads per KV head handled by one WG
// The reference of a query's weights 2^(s - ref), in the log2 domain.  P enters
// P V rounded to bf16, and a weight that is a power of two does not round; so
// the heaviest weights, those that make a row, round least if the references
// have the fractions of the maxima of many tiles.  With one running maximum per
// range the error therefore grows with the range's length (rms of the weights'
// part over 512, 8224 and 32800 normal keys: 1.42, 1.59 and 1.63e-3).  So a tile
// may restart the reference at its own maximum, moved up by whole powers of two
// to at least the maximum so far (no accumulator grows), and in between a
// larger maximum raises it.  A restart costs a rescale of the accumulators.
// Where a maximum is young, tiles rescale anyway (some of a wave's 32 queries
// rises in two of three tiles up to the 32nd): there every tile restarts, later
// every fourth (1.17 and 1.54e-3: less than any range of a quarter or an eighth of
// the length, which is how much shorter equal cuts of the longest prefix are).
// The register-staged kernel, which waits for its own arithmetic, restarts at
// every second of the early tiles (1.41e-3).
// Error against 64 bits, bf16 outputs included, and time of 128 x 32768 keys:
// 2.25e-3 and 1531 us, with one running maximum per range 2.32e-3 and 1528 us,
// with a restart at every tile throughout 2.1e-3 and 1710 us; 24 paged requests
// of 1 to 8192: 2.0e-3 and 70 us, and 2.2e-3 and 71 us.
struct SpRef {
  float most = -INFINITY;  // maximum so far
  float ref = -INFINITY;
  template <int kEarly>
  __device__ static inline bool restarts(int n) { return n < 64 ? n % kEarly == 0 : n % 4 == 0; }
  // Takes a tile's maximum; true where some lane's reference moves, to next
  // (what it was is left in ref for the rescale, and set by the caller).
  __device__ inline bool take(float mt, bool restart, float& next) {
    most = fmaxf(most, mt);
    const float w = fmaxf(mt, most - 100.0f);  // (finite after a finite tile)
    const float anew = w + fmaxf(0.0f, ceilf(most - w)), on = fmaxf(ref, mt);
    // A select although restart is uniform: with a branch, the wait states between
    // P V and the rescale were counted along the longer way (mma_settle).
    next = restart ? anew : on;
    return __any(next != ref);
  }
};

// One wave per query head of the KV group; 32-key tiles double-buffered in
// LDS: the tile after next is loaded into registers while the current one is
// computed, and the next one is moved from registers into the free buffer at
// the end of the step, so one barrier per tile orders everything.
template <typename T, int D, int NG, bool PAGED, bool WIN = false>
__global__ __launch_bounds__(kWave* NG) void hyb_sp_partial_kernel(
    SoftmaxPrefixArgs a, SpCut cut) {
  typedef SpCfg<T, D, NG> C;
  typedef typename C::M M;
  typedef typename C::op_t op_t;
  constexpr int E = M::E, KW = M::KW, EPC = C::EPC, CPR = C::CPR, NCH = C::NCH;
  __shared__ typename C::Smem sh;

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L, G = Hq / Hkv;
  const int Pmax = a.max_prefix;
  const int g = blockIdx.x % Hkv, r = blockIdx.x / Hkv, h = g * G + w;
  static_assert(sizeof(sh.v[1]) >= kPlanInts * sizeof(int), "the plan's scratch fits a tile");
  const SpRange rg = sp_range<WIN>(a, sp_plan<WIN>(a, cut, reinterpret_cast<int*>(sh.v[1])), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int b = rg.b, lo = rg.lo, hi = rg.hi;
  const int Lb = sp_block<WIN>(a, b);  // active queries
  const int P = sp_keys<WIN>(a, b) - Lb;
  const SpSeen seen = sp_seen<WIN>(a, b);
  const size_t qstride = (size_t)Hq * D, kstride = (size_t)Hkv * D;

  op_t qop[C::KD];
  {
    const T* qrow = (const T*)a.q + ((size_t)b * L * Hq + h) * D +
                    (size_t)li * qstride + hh * E;
#pragma unroll
    for (int ks = 0; ks < C::KD; ++ks)
      qop[ks] = li < Lb ? load_op<T>(qrow + ks * KW) : M::zero();
  }
  // contiguous: this request's rows; paged: the pool, at KV head g
  const T* kc = (const T*)a.k_cache + ((PAGED ? 0 : (size_t)b * Pmax * Hkv) + g) * D;
  const T* vc = (const T*)a.v_cache + ((PAGED ? 0 : (size_t)b * Pmax * Hkv) + g) * D;
  const T* kbk = (const T*)a.k + ((size_t)b * L * Hkv + g) * D;
  const T* vbk = (const T*)a.v + ((size_t)b * L * Hkv + g) * D;
  const int32_t* ptab = PAGED ? a.page_table + (size_t)b * a.max_pages : nullptr;
  // row offset of cached token j (j < P)
  auto crow = [&](int j) __attribute__((always_inline)) -> size_t {
    if constexpr (PAGED)
      return (((size_t)sp_page(a, ptab, j) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) *
             kstride;
    else
      return (size_t)j * kstride;
  };

  // Tile loads: keys past the range read the range's last key (in bounds)
  // and are masked out of the scores below.
  // A tile's share of this thread, held in registers between its load and
  // its move into LDS: nx is the next tile, af the one after it.
  struct TileRegs {
    uint4 k[NCH], v[NCH];
  };
  auto fetch = [&](int j0) __attribute__((always_inline)) {
    TileRegs r;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int idx = tid + c * kWave * NG, key = idx / CPR, part = idx % CPR;
      if (idx < kTile * CPR) {  // (NG not a power of two: a partial last set)
        int j = min(j0 + key, hi - 1);
        if constexpr (WIN) j = seen.hides(j) ? seen.stand_in(j0) : j;
        const size_t o = (size_t)part * EPC;
        const size_t cr = j < P ? crow(j) : 0;
        const T* ks = j < P ? kc + cr : kbk + (size_t)(j - P) * kstride;
        const T* vs = j < P ? vc + cr : vbk + (size_t)(j - P) * kstride;
        r.k[c] = *reinterpret_cast<const uint4*>(ks + o);
        r.v[c] = *reinterpret_cast<const uint4*>(vs + o);
      }
    }
    return r;
  };
  auto put = [&](const TileRegs& r, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int idx = tid + c * kWave * NG, key = idx / CPR, part = idx % CPR;
      if (idx < kTile * CPR) {
        *reinterpret_cast<uint4*>(&sh.k[buf][key][part * EPC]) = r.k[c];
        *reinterpret_cast<uint4*>(&sh.v[buf][key][part * EPC]) = r.v[c];
      }
    }
  };
  // V^T operand of column tile ct, k-step ks: lane (li, hh) holds column
  // ct*32 + li at keys row_of(ks*E + e, hh).  bf16: in each 16-lane quarter
  // the transposing read gives lane i element i%4 of the 8-byte pieces
  // addressed by lanes i/4 + 4j (j = 0..3); lane i addresses key
  // kb + i/4 at columns cb + 4*(i%4) .. +3, so it receives keys kb .. kb+3
  // of column cb + i.
  auto vt_op = [&](int buf, int ct, int ks) __attribute__((always_inline)) -> op_t {
    if constexpr (E == 1) {
      return to_f32(sh.v[buf][row_of(ks, hh)][ct * kTile + li]);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const int i = lane & 15;
      const int cb = ct * kTile + 16 * ((lane >> 4) & 1);
      const int kb = 16 * ks + 4 * hh;
      auto piece = [&](int key) {
        const T* src = &sh.v[buf][key][cb + 4 * (i & 3)];
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)src);
      };
      const s16x4 x0 = piece(kb + i / 4), x1 = piece(kb + 8 + i / 4);
      return __builtin_bit_cast(op_t, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };

  // Scores are scaled by 1/sqrt(d) and, on bf16, kept in the log2 domain of
  // SpRef (fp32 weights do not round, and keep one running maximum).
  constexpr bool kWin = sizeof(T) == 2;
  const float scale = (kWin ? kLog2e : 1.0f) / sqrtf((float)D);
  SpRef rf;
  float& m = rf.ref;
  float l = 0.0f;
  f32x16 acc[C::NCT];
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) acc[ct] = f32x16{};

  // First key of the tile x tiles after the one at j0, the range's n-th.
  auto after = [&](int j0, int n, int x) __attribute__((always_inline)) {
    return WIN ? (n + x < rg.nt ? seen.tile(rg.t0 + n + x) * kTile : hi) : j0 + x * kTile;
  };
  TileRegs nx = {}, af = {};
  if (lo < hi) {
    put(fetch(lo), 0);
    if (after(lo, 0, 1) < hi) nx = fetch(after(lo, 0, 1));
  }
  __syncthreads();
  int n = 0;
  for (int j0 = lo; j0 < hi; j0 = after(j0, n, 1), ++n) {
    const int buf = n & 1;
    if (after(j0, n, 2) < hi) af = fetch(after(j0, n, 2));  // tile after next

    f32x16 sc = {};
#pragma unroll
    for (int ks = 0; ks < C::KD; ++ks)
      sc = M::mma(load_op<T>(&sh.k[buf][li][ks * KW + hh * E]), qop[ks], sc);
    if constexpr (WIN) mma_settle<T>();
    // Scaled scores; keys past the range only in the range's last tile
    // (a wave-uniform test, so full tiles carry no masks).
    const bool full = j0 + kTile <= hi && !(WIN && seen.cuts(j0));
    float p[16];
    float mt = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = j0 + row_of(i, hh);
      p[i] = (full || (j < hi && !(WIN && seen.hides(j)))) ? sc[i] * scale : -INFINITY;
      mt = fmaxf(mt, p[i]);
    }
    mt = fmaxf(mt, xor32(mt));
    float mn;
    bool moves;
    if constexpr (kWin) {
      moves = rf.take(mt, SpRef::restarts<2>(n), mn);
    } else {
      mn = fmaxf(m, mt);
      moves = __any(mn > m);
    }
    auto ex = [](float x) { return kWin ? __builtin_amdgcn_exp2f(x) : fast_exp(x); };
    float ps = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = as_operand<T>(ex(p[i] - mn));  // exp(-inf) = 0 past the range
      ps += p[i];
    }
    ps += xor32(ps);
    // The accumulators are rescaled only when some query's reference moved:
    // once the maximum settles most tiles skip the 64 multiplies.
    if (moves) {
      const float corr = ex(m - mn);
      l *= corr;
#pragma unroll
      for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[ct][i] *= corr;
    }
    l += ps;
    m = mn;
#pragma unroll
    for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
      for (int ks = 0; ks < C::KL; ++ks)
        acc[ct] = M::mma(vt_op(buf, ct, ks), cvt_op<T>(&p[ks * E]), acc[ct]);
    if constexpr (WIN) mma_settle<T>();
    if (after(j0, n, 1) < hi) put(nx, buf ^ 1);  // next tile into the free buffer
    // (the next step may move the sums between registers before it branches)
    if constexpr (!WIN && sizeof(T) == 4) mma_settle<T>();
    nx = af;
    __syncthreads();
  }

  // Partial result of this range: unnormalised O, running max and sum.
  mma_settle<T>();
  if (li >= Lb) return;
  if (rg.n == 1) {
    // one range: the result is final, normalised here
    const float inv = 1.0f / l;
    const size_t ob = (((size_t)b * L + li) * Hq + h) * D;
#pragma unroll
    for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float o[4] = {acc[ct][i] * inv, acc[ct][i + 1] * inv, acc[ct][i + 2] * inv,
                            acc[ct][i + 3] * inv};
        store_out4<T>(a.out, ob + ct * kTile + row_of(i, hh), o, a.s.out_f32);
      }
    return;
  }
  const size_t row = sp_row(a, r, h, li);
  float* wacc = (float*)a.ws + row * D;
  float* wml = sp_ml<D>(a) + row * 2;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<f32x4*>(wacc + ct * kTile + row_of(i, hh)) =
          f32x4{acc[ct][i], acc[ct][i + 1], acc[ct][i + 2], acc[ct][i + 3]};
  if (hh == 0) {
    wml[0] = kWin ? m * 0.6931471805599453f : m;  // (the natural log)
    wml[1] = l;
  }
}


// bf16 with 1, 2, 4 or 8 query heads per KV head: the K and V tiles reach
// LDS by direct global->LDS copies into two rings of R = 4 tile slots, three
// tiles in flight while one is computed, with no registers held for them.
// Each copy instruction reads whole rows, 16 bytes per lane; chunk c of a
// staged K row t sits at position c ^ swz(t), of a V row at c ^ vswz(t), so
// the rows one operand read touches fall in distinct LDS banks (a K operand
// reads one chunk of 32 rows, a transposing V read four chunks of 4 rows per
// half wave).  The slots are distinct arrays and the
// tile loop is unrolled over them, so every copy and every read names its
// slot at compile time.  A wave waits only for its own copies of the tiles it
// is about to read (vmcnt counts the later tiles' copies still in flight),
// then one barrier per tile makes all of them visible and frees the slots the
// next copies reuse.
//
// What bounds the loop is each wave's chain, not the copies: scores (8
// dependent MFMAs), maximum, exponentials, P V (8 MFMAs).  So step n forms
// the scores of tile n + 1 while it takes the softmax of tile n: two
// independent chains whose MFMAs and VALU instructions interleave.  That is
// why K runs one tile ahead of V in its ring.  At 128 requests of 32768 keys:
// 1.72 ms (5.0 TB/s) as one chain, 1.51 ms (5.7 TB/s) so.
template <int D>
struct SpRing {
  static constexpr int EPC = 8;                      // bf16 per 16 bytes
  static constexpr int CPR = D / EPC;                // chunks per row
  static constexpr int RPI = kWave / CPR;            // rows per copy instruction
  static constexpr int RP256 = 256 / (D * 2) > 0 ? 256 / (D * 2) : 1;
  static constexpr int IK = kTile / RPI;             // copies per 32-row tile
  static constexpr int R = 4;                        // ring slots
  __device__ static constexpr int swz(int t) { return (t / RP256) % CPR; }
  __device__ static constexpr int vswz(int t) { return 4 * ((t / RP256) % (CPR / 4)); }
};

// c ? a : b of values: written out over two captured variables it is a choice of
// their addresses, which can leave a lambda's captures in scratch memory.
__device__ inline const bf16* sp_pick(bool c, const bf16* a, const bf16* b) { return c ? a : b; }

template <int D>
struct alignas(16) SpSlot {
  bf16 k[kTile * D];
  bf16 v[kTile * D];
};

template <int D, int NG, bool PAGED, bool WIN = false>
__global__ __launch_bounds__(kWave* NG, D == 64 && NG == 8 ? 4 : 2) void hyb_sp_ring_kernel(SoftmaxPrefixArgs a, SpCut cut) {
  typedef Mma<bf16> M;
  typedef typename M::op_t op_t;
  typedef SpRing<D> RG;
  constexpr int E = M::E, KW = M::KW, KD = D / KW, KL = kTile / KW, NCT = D / kTile;
  constexpr int EPC = RG::EPC, CPR = RG::CPR, RPI = RG::RPI, IK = RG::IK, R = RG::R;
  constexpr int IPW = 2 * IK / NG;  // copies per wave and step
  static_assert(IPW * NG == 2 * IK, "copies split evenly over the waves");
  static_assert(3 * IPW <= 63, "a wave's copies in flight fit vmcnt");
  __shared__ SpSlot<D> s0, s1, s2, s3;

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L, G = Hq / Hkv;
  const int Pmax = a.max_prefix;
  // The KV head varies fastest: the Hkv workgroups that read the same
  // token rows of the cache (each its 1/Hkv share of every row) start
  // together.
  const int g = blockIdx.x % Hkv, r = blockIdx.x / Hkv, h = g * G + w;
  static_assert(sizeof(s3.v) >= kPlanInts * sizeof(int), "the plan's scratch fits a tile");
  const SpRange rg = sp_range<WIN>(a, sp_plan<WIN>(a, cut, reinterpret_cast<int*>(s3.v)), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int b = rg.b, lo = rg.lo, hi = rg.hi;
  const int Lb = sp_block<WIN>(a, b);  // active queries
  const int P = sp_keys<WIN>(a, b) - Lb;
  const SpSeen seen = sp_seen<WIN>(a, b);
  const int ntiles = WIN ? rg.nt : (hi - lo + kTile - 1) / kTile;
  const size_t qstride = (size_t)Hq * D, kstride = (size_t)Hkv * D;

  op_t qop[KD];
  {
    const bf16* qrow =
        (const bf16*)a.q + ((size_t)b * L * Hq + h) * D + (size_t)min(li, Lb - 1) * qstride + hh * E;
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) qop[ks] = keep_if<bf16>(li < Lb, load_op<bf16>(qrow + ks * KW));
  }
  // contiguous: this request's rows; paged: the pool, at KV head g
  const bf16* kc = (const bf16*)a.k_cache + ((PAGED ? 0 : (size_t)b * Pmax * Hkv) + g) * D;
  const bf16* vc = (const bf16*)a.v_cache + ((PAGED ? 0 : (size_t)b * Pmax * Hkv) + g) * D;
  const bf16* kbk = (const bf16*)a.k + ((size_t)b * L * Hkv + g) * D;
  const bf16* vbk = (const bf16*)a.v + ((size_t)b * L * Hkv + g) * D;
  // Paged: the pages of the cached keys of this range, lo .. min(hi, P) - 1,
  // staged in LDS (page index p0 + e at e; behind page pa, the last before the
  // skipped tiles, p0 + e + pskip), clamped to the pool.
  __shared__ int pages[PAGED ? kMaxRangePages : 1];
  const int p0 = lo >> a.page_shift;
  int pa = 0x7fffffff, pskip = 0;
  if constexpr (WIN) {
    if (seen.skip > 0 && rg.t0 < seen.st && rg.t0 + rg.nt > seen.st) {
      pa = (seen.st * kTile - 1) >> a.page_shift;
      pskip = max(0, ((seen.st + seen.skip) * kTile >> a.page_shift) - pa - 1);
    }
  }
  auto page_of = [&](int pi) __attribute__((always_inline)) {
    return pages[pi - p0 - (WIN && pi > pa ? pskip : 0)];
  };
  if constexpr (PAGED) {
    const int32_t* ptab = a.page_table + (size_t)b * a.max_pages;
    const int chi = min(hi, P);
    const int np = chi > lo ? ((chi - 1) >> a.page_shift) - p0 + 1 - pskip : 0;
    for (int e = tid; e < np; e += kWave * NG) {
      const int pi = p0 + e + (WIN && p0 + e > pa ? pskip : 0);
      pages[e] = sp_page(a, ptab, pi << a.page_shift);
    }
    __syncthreads();
  }

  // Copies of a tile that lies wholly in the cached prefix: a buffer
  // descriptor whose base is the tile's first row (a scalar) and, per lane
  // and copy, the 32-bit offset of its 16-byte piece, which is the same for
  // every tile.  Tiles that reach past the cache or the range take the
  // general path below.  Copy ins of a step is K's (kv = 0) or V's (kv = 1);
  // a wave's copies are all of one kind, except with one wave (NG = 1).
  int voff[IPW];
#pragma unroll
  for (int u = 0; u < IPW; ++u) {
    const int ins = w * IPW + u, i = ins % IK;
    const int t = i * RPI + lane / CPR, pos = lane % CPR;
    const int sw = ins < IK ? RG::swz(t) : RG::vswz(t);
    voff[u] = (int)(((size_t)t * kstride + (size_t)((pos ^ sw) * EPC)) * sizeof(bf16));
  }
  const int cend = min(hi, P);  // keys below this come from the cache
  // The order of the tiles.  Those that reach past the cache (the range's last
  // one or two, nlate of them: a block is at most a tile long) come first, the last
  // one foremost: their copies are all issued before the loop, and only tile 0
  // can be partial, so the loop's steps need neither the general copies nor
  // masks.  (With them last and a second set of steps for the last tiles the
  // code was twice as long, and a short range, which runs it once, waited for its
  // instructions: with one head per KV head at d = 128 one request of 300 keys
  // took 21.4 us, now 15.7, 32 of 512 28.1 and 24.1, 32 of 4096 138 and 115.)
  // With WIN (every tile of the list is one of the whole, 32-aligned tiles of
  // the keys) those wholly in the cache are the tiles below P / 32.
  const int nlate =
      WIN ? ntiles - min(max(P / kTile - seen.skip - rg.t0, 0), ntiles) : ntiles - (cend > lo ? (cend - lo) / kTile : 0);
  auto first_key = [&](int n) __attribute__((always_inline)) {
    const int i = n < nlate ? ntiles - 1 - n : n - nlate;
    return WIN ? seen.tile(rg.t0 + i) * kTile : lo + i * kTile;
  };
  constexpr int NKV = NG == 1 ? 2 : 1;      // kinds of copies per wave
  constexpr int IPK = IPW / NKV;            // copies per kind
  // This wave's copies u0 .. u0 + IPK - 1, of kind kv, of tile n into dst.
  auto issue_cached = [&](int kv, int u0, int n, bf16* dst) __attribute__((always_inline)) {
    const int j0 = WIN ? first_key(n) : lo + (n - nlate) * kTile;
    const bf16* cb = sp_pick(kv == 0, kc, vc);
    if constexpr (PAGED) {
      const int pi = j0 >> a.page_shift;
      cb += ((ptrdiff_t)__builtin_amdgcn_readfirstlane(page_of(pi)) - pi) *
            ((ptrdiff_t)kstride << a.page_shift);
    }
    cb += (size_t)j0 * kstride;
    const int span = (int)((size_t)kTile * kstride * sizeof(bf16));
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(cb), 0, span, kBufferWord3);
#pragma unroll
    for (int u = u0; u < u0 + IPK; ++u) buf_to_lds16(rs, dst + (w * IPW + u) % IK * RPI * D, voff[u], 0);
  };
  // The same of a tile that reaches past the cache (keys past the range read
  // the range's last key, in bounds, and are masked below).
  auto issue_general = [&](int kv, int u0, int n, bf16* dst) __attribute__((always_inline)) {
    const int j0 = first_key(n);
    const bf16* cb = sp_pick(kv == 0, kc, vc);
    if constexpr (PAGED) {
      // the tile's rows (clamped to the range, all >= j0) lie in the page of
      // row j0: that page's base, shifted so that base + j * kstride is row j
      if (j0 < P) {
        const int pi = j0 >> a.page_shift;
        cb += ((ptrdiff_t)page_of(pi) - pi) * ((ptrdiff_t)kstride << a.page_shift);
      }
    }
    const bf16* blk = sp_pick(kv == 0, kbk, vbk);
#pragma unroll
    for (int u = u0; u < u0 + IPK; ++u) {
      const int i = (w * IPW + u) % IK;
      const int t = i * RPI + lane / CPR, pos = lane % CPR;
      int j = min(j0 + t, hi - 1);
      if constexpr (WIN) j = seen.hides(j) ? seen.stand_in(j0) : j;
      const bf16* row = sp_pick(j < P, cb, blk) + (size_t)(j < P ? j : j - P) * kstride;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(row + (pos ^ (kv == 0 ? RG::swz(t) : RG::vswz(t))) * EPC),
          (__attribute__((address_space(3))) void*)(dst + i * RPI * D), 16, 0, 0);
    }
  };
  // The copies of step n: K of tile nk and V of tile nv, where they exist
  // (early: tiles 0 and 1, which may reach past the cache).
  auto issue = [&](auto early, int nk, SpSlot<D>& sk, int nv, SpSlot<D>& sv) __attribute__((always_inline)) {
    auto one = [&](int kv, int u0, int n, bf16* dst) __attribute__((always_inline)) {
      if constexpr (decltype(early)::value || WIN) {
        if (n < nlate || (WIN && seen.cuts(first_key(n)))) {
          issue_general(kv, u0, n, dst);
          return;
        }
      }
      issue_cached(kv, u0, n, dst);
    };
    if constexpr (NG == 1) {
      if (nk < ntiles) one(0, 0, nk, sk.k);
      if (nv >= 0 && nv < ntiles) one(1, IPK, nv, sv.v);
    } else {
      const int kv = w * IPW / IK, n = kv == 0 ? nk : nv;
      if (n >= 0 && n < ntiles) one(kv, 0, n, kv == 0 ? sk.k : sv.v);
    }
  };

  // Scores and the reference m (SpRef) are kept in the log2 domain (scaled by
  // log2 e with 1/sqrt(d)), so each weight is one fma and one exp2;
  // m is converted back where it is written out for the combine.
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  // The running sum of the weights comes from the MFMAs, so it is the sum of
  // the same rounded weights that enter P V: a 16x16 product whose column
  // li % 16 holds, as its contraction quarters, the keys of queries li % 16
  // (even quarters) and li % 16 + 16 (odd ones).  Row x of the left operand
  // is one on the quarters of the parity of x / 4, which is that of the lane
  // that receives the row, so register 0 is the sum of the lane's own query
  // (only that register is kept rescaled).
  SpRef rf;
  float& m = rf.ref;
  f32x16 acc[NCT];
  f32x4 lsum = {};
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  op_t ones;
#pragma unroll
  for (int e = 0; e < E; ++e) ones[e] = (bf16)(((lane >> 4) ^ (lane >> 2)) & 1 ? 0.0f : 1.0f);

  // Raw scores of a tile: keys in rows, queries in columns.
  auto k_op = [&](const bf16* kt, int ks) __attribute__((always_inline)) -> op_t {
    const int c = 2 * ks + hh;  // 16-byte chunk of elements ks*KW + hh*E
    return load_op<bf16>(&kt[li * D + (c ^ RG::swz(li)) * EPC]);
  };
  // Scores of the tile of the current step, already in the reference (and the
  // accumulators rescaled to it).
  f32x16 sc;
  // Takes the scores of tile n into sc and the reference.  The accumulators are
  // rescaled only when some query's reference moved: once the maximum settles
  // most tiles skip the 64 multiplies.  Keys past the range, in tile 0 only,
  // are masked.
  auto take_scores = [&](auto check, int n, const f32x16& s) __attribute__((always_inline)) {
    sc = s;
    if constexpr (decltype(check)::value || WIN) {
      if constexpr (WIN) mma_settle<bf16>();
      const int j0 = first_key(n);
      if (j0 + kTile > hi || (WIN && seen.cuts(j0))) {  // uniform
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = j0 + row_of(i, hh);
          sc[i] = j < hi && !(WIN && seen.hides(j)) ? sc[i] : -INFINITY;
        }
      }
    }
    float mt = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sc[i]);
    mt = fmaxf(mt, xor32(mt));
    float mn;
    if (rf.take(mt * scale, SpRef::restarts<1>(n), mn)) {
      if constexpr (WIN) mma_settle<bf16>();
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      lsum[0] *= corr;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[ct][i] *= corr;
    }
    m = mn;
  };

  // Weights and P V of tile n (its scores in sc, its V in vt) and the scores
  // of tile n + 1 (its K in kt; not with LAST), then that tile's maximum.
  auto compute = [&](auto last, int n, const bf16* kt, const bf16* vt) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(last)::value;
    op_t kop[KD];
    if constexpr (!LAST) {
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) kop[ks] = k_op(kt, ks);
    }
    f32x16 sn = {};
    if constexpr (!LAST) {
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) sn = M::mma(kop[ks], qop[ks], sn);
    }
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], scale, -m));
    op_t pop[KL];
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) pop[ks] = cvt_op<bf16>(&p[ks * E]);
    // V^T operands by transposing reads: in each 16-lane quarter lane i
    // addresses key kb + i/4 at columns cb + 4*(i%4) .. +3 and receives
    // keys kb .. kb+3 of column cb + i.
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const int qi = lane & 15;
    op_t vop[NCT][KL];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      const int col = ct * kTile + 16 * ((lane >> 4) & 1) + 4 * (qi & 3);
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) {
        auto piece = [&](int t) {
          // (t = kb + 8n: vswz(t) is that of the lane's qi / 4)
          const bf16* src = &vt[t * D + ((col / EPC) ^ RG::vswz(qi / 4)) * EPC + col % EPC];
          return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)src);
        };
        const int kb = 16 * ks + 4 * hh + qi / 4;
        const s16x4 x0 = piece(kb), x1 = piece(kb + 8);
        vop[ct][ks] = __builtin_bit_cast(op_t, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) acc[ct] = M::mma(vop[ct][ks], pop[ks], acc[ct]);
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) lsum = Mma16<bf16>::mma(ones, pop[ks], lsum);
    if constexpr (!LAST) {
      // The order of issue: K's operands; the score MFMAs with the weights
      // between them, V's operands requested behind the first half of them;
      // then P V with the next tile's maximum.
      __builtin_amdgcn_sched_group_barrier(0x100, KD, 0);  // LDS reads
#pragma unroll
      for (int ks = 0; ks < KD / 2; ++ks) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // an MFMA
        __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);  // VALU, exp
      }
#pragma unroll
      for (int ks = KD / 2; ks < KD; ++ks) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4 * NCT * KL / KD, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);
      }
      take_scores(std::false_type{}, n + 1, sn);
    }
  };

  // Wait for this wave's copies of the tiles of a step, with at most `later`
  // steps' copies issued after them still in flight.
  auto wait_step = [&](int later) __attribute__((always_inline)) {
    if (later >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * IPW) : "memory");
    else if (later == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * IPW) : "memory");
    else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPW) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  };
  auto slot = [&](auto S) -> SpSlot<D>& {
    if constexpr (decltype(S)::value == 0) return s0;
    else if constexpr (decltype(S)::value == 1) return s1;
    else if constexpr (decltype(S)::value == 2) return s2;
    else return s3;
  };
  // A wave's last tile whose copies it must see: V's wave n, K's wave n + 1.
  // With one wave, a step's copies are K n + 1 and V n; whole steps are
  // counted while both kinds are still issued.
  const int ahead = NG == 1 || w * IPW / IK == 0 ? 1 : 0;
  auto step = [&](int n, auto S) __attribute__((always_inline)) {
    constexpr int SV = decltype(S)::value;
    const int later = ntiles - 1 - n - ahead;
    if constexpr (NG == 1) wait_step(later >= 2 ? 2 : 0);
    else wait_step(min(2, later));
    lds_barrier_nodrain();  // K n+1 and V n visible everywhere; K n's and V n-1's slots free
    issue(std::false_type{}, n + R, slot(S), n + R - 1, slot(std::integral_constant<int, (SV + R - 1) % R>{}));
    compute(std::false_type{}, n, slot(std::integral_constant<int, (SV + 1) % R>{}).k, slot(S).v);
  };

  // Copies of K 0 .. R-1 and V 0 .. R-2, in the order of the steps' copies.
  const std::true_type yes{};
  issue(yes, 0, s0, -1, s0);
  issue(yes, 1, s1, 0, s0);
  issue(yes, 2, s2, 1, s1);  // (K of tile 2 is a cached tile's)
  issue(std::false_type{}, 3, s3, 2, s2);
  if constexpr (NG == 1) wait_step(ntiles >= R ? 3 : 0);
  else wait_step(ahead ? min(3, ntiles - 1) : 3);  // (V's waves need nothing yet)
  lds_barrier_nodrain();
  {
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) s = M::mma(k_op(s0.k, ks), qop[ks], s);
    take_scores(yes, 0, s);
  }
  int n = 0;
  for (; n + R < ntiles; n += R) {
    step(n, std::integral_constant<int, 0>{});
    step(n + 1, std::integral_constant<int, 1>{});
    step(n + 2, std::integral_constant<int, 2>{});
    step(n + 3, std::integral_constant<int, 3>{});
  }
  if (n + 1 < ntiles) step(n, std::integral_constant<int, 0>{});
  if (n + 2 < ntiles) step(n + 1, std::integral_constant<int, 1>{});
  if (n + 3 < ntiles) step(n + 2, std::integral_constant<int, 2>{});
  // the last tile: every copy has landed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_barrier_nodrain();
  const int rest = ntiles - n;  // 1 .. R
  compute(yes, ntiles - 1, nullptr, rest == 2 ? s1.v : rest == 3 ? s2.v : rest == 4 ? s3.v : s0.v);
  mma_settle<bf16>();

  if (li >= Lb) return;
  const float l = lsum[0];
  if (rg.n == 1) {
    // one range: the result is final, normalised here
    const float inv = 1.0f / l;
    const size_t ob = (((size_t)b * L + li) * Hq + h) * D;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float o[4] = {acc[ct][i] * inv, acc[ct][i + 1] * inv, acc[ct][i + 2] * inv,
                            acc[ct][i + 3] * inv};
        store_out4<bf16>(a.out, ob + ct * kTile + row_of(i, hh), o, a.s.out_f32);
      }
    return;
  }
  const size_t row = sp_row(a, r, h, li);
  float* wacc = (float*)a.ws + row * D;
  float* wml = sp_ml<D>(a) + row * 2;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<f32x4*>(wacc + ct * kTile + row_of(i, hh)) =
          f32x4{acc[ct][i], acc[ct][i + 1], acc[ct][i + 2], acc[ct][i + 3]};
  if (hh == 0) {
    wml[0] = m * 0.6931471805599453f;  // back to the natural log
    wml[1] = l;
  }
}

// ---- kernels of a window ------------------------------------------------------
//
// A range's tiles for a workgroup of the kernels below: where they are and how a
// wave copies rows of one.  `pages` is LDS for kMaxRangePages numbers.
template <int D>
struct SpTiles {
  typedef RowColTile<D> RT;
  const bf16 *kc, *vc, *kb, *vb;  // cache pools and block at the KV head
  SpSeen seen;
  int t0, nt, hi, P, page_shift, p0, pa, pskip;
  int kstride;  // elements from a token to the next
  const int* pages;

  // All threads of the workgroup; ends with a barrier.
  __device__ inline SpTiles(const SoftmaxPrefixArgs& a, const SpRange& rg, int g, int P_, int* lds) {
    kc = (const bf16*)a.k_cache + g * D;
    vc = (const bf16*)a.v_cache + g * D;
    kb = (const bf16*)a.k + ((size_t)rg.b * a.s.L * a.s.Hkv + g) * D;
    vb = (const bf16*)a.v + ((size_t)rg.b * a.s.L * a.s.Hkv + g) * D;
    seen = sp_seen<true>(a, rg.b);
    t0 = rg.t0, nt = rg.nt, hi = rg.hi, P = P_;
    page_shift = a.page_shift;
    kstride = a.s.Hkv * D;
    pages = lds;
    // the pages of the range's cached keys, as in the ring kernel
    p0 = rg.lo >> page_shift;
    pa = 0x7fffffff;
    pskip = 0;
    if (seen.skip > 0 && t0 < seen.st && t0 + nt > seen.st) {
      pa = (seen.st * kTile - 1) >> page_shift;
      pskip = max(0, ((seen.st + seen.skip) * kTile >> page_shift) - pa - 1);
    }
    const int32_t* ptab = a.page_table + (size_t)rg.b * a.max_pages;
    const int chi = min(hi, P);
    const int np = chi > rg.lo ? ((chi - 1) >> page_shift) - p0 + 1 - pskip : 0;
    for (int e = threadIdx.x; e < np; e += blockDim.x)
      lds[e] = sp_page(a, ptab, (p0 + e + (p0 + e > pa ? pskip : 0)) << page_shift);
    __syncthreads();
  }
  // First key of the range's tile i.
  __device__ inline int first_key(int i) const { return seen.tile(t0 + i) * kTile; }
  // This lane's row and entry in copy u of a tile.
  __device__ static inline int copy_row(int u, int lane) { return u * RT::RPI + lane / RT::CPR; }
  __device__ static inline int copy_col(int u, int lane) {
    return (lane % RT::CPR ^ RT::swz(copy_row(u, lane))) * RT::EPC;
  }
  // Copies u0 .. u0 + N - 1 of K (kv = 0) or V of the tile at j0 into dst.
  template <int N>
  __device__ inline void copy(int kv, int j0, int u0, bf16* dst, int lane) const {
    ptrdiff_t shift = 0;  // from a row's place in its request to its place in the pools
    if (j0 < P) {
      const int pi = j0 >> page_shift;
      shift = ((ptrdiff_t)__builtin_amdgcn_readfirstlane(pages[pi - p0 - (pi > pa ? pskip : 0)]) - pi) << page_shift;
    }
    if (j0 + kTile <= min(hi, P) && !seen.cuts(j0)) {  // uniform: wholly in the cache and seen
      const bf16* base = sp_pick(kv == 0, kc, vc) + (shift + j0) * (ptrdiff_t)kstride;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<bf16*>(base), 0, (int)(kTile * kstride * sizeof(bf16)), kBufferWord3);
#pragma unroll
      for (int u = 0; u < N; ++u)
        buf_to_lds16(rs, dst + (u0 + u) * RT::RPI * D,
                     (int)((copy_row(u0 + u, lane) * kstride + copy_col(u0 + u, lane)) * sizeof(bf16)), 0);
    } else {
      // keys past the range and hidden ones read a visible row of the tile
#pragma unroll
      for (int u = 0; u < N; ++u) {
        int j = min(j0 + copy_row(u0 + u, lane), hi - 1);
        j = seen.hides(j) ? seen.stand_in(j0) : j;
        const bf16* base = sp_pick(j < P, sp_pick(kv == 0, kc, vc), sp_pick(kv == 0, kb, vb));
        const bf16* row = base + (ptrdiff_t)(j < P ? shift + j : j - P) * kstride + copy_col(u0 + u, lane);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)row,
                                         (__attribute__((address_space(3))) void*)(dst + (u0 + u) * RT::RPI * D), 16, 0, 0);
      }
    }
  }
};

// What a wave keeps of its 32 columns (queries): the weights' reference in the
// log2 domain (finite, so that a wave without tiles weighs nothing; it moves only
// when a maximum passes it by 2^8), their sum over the lane's rows, and the
// weighted sums of V^T.
template <int D>
struct SpAcc {
  typedef Mma<bf16> M;
  static constexpr int KD = D / M::KW, KL = kTile / M::KW, NCT = D / kTile;
  float m = -1e30f, l = 0.0f;
  f32x16 acc[NCT];
  __device__ inline SpAcc() {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  }
  // Adds the tile at j0 (K, V in LDS); scale = log2(e) / sqrt(d).
  __device__ inline void add(const SpTiles<D>& t, const RowColTile<D>& rt, int j0, const bf16* kt, const bf16* vt,
                             const bf16x8 (&qop)[KD], float scale, int hh) {
    f32x16 sc = {};
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) sc = M::mma(rt.row_op(kt, ks), qop[ks], sc);
    mma_settle<bf16>();
    if (j0 + kTile > t.hi || t.seen.cuts(j0)) {  // uniform
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = j0 + row_of(e, hh);
        sc[e] = j < t.hi && !t.seen.hides(j) ? sc[e] : -INFINITY;
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
    // The weights enter P V rounded to bf16 (each off by at most 2^-8 of itself;
    // products of fp32 run at 1/16 of the rate); their sum is over the unrounded ones.
    bf16x8 pop[KL];
    float sum[4] = {};
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[ks * 8 + e], scale, -m));
        sum[e % 4] += p[e];
      }
      pop[ks] = cvt_op<bf16>(p);
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) acc[ct] = M::mma(rt.col_op(vt, ct, ks), pop[ks], acc[ct]);
  }
};

// Few queries (bf16; decoding, and small batches of blocks): as many of a KV
// head's query heads as have their L queries within the 32 columns of one tile of
// scores share a workgroup (all of them in decoding), a wave answers all columns,
// and the four waves take the range's tiles in turn, each with copies of its own
// (two slots of K and V, no barrier in the loop) and sums of its own, joined in
// LDS at the end.  With a wave per head, as above, each has one or a few columns of
// its tile filled, and the loop is four times as many dependent steps (one token
// of 64 requests over a window of 4096 117 us, now 98; of one request 25 and 17).
__host__ __device__ inline int sp_pack(const Shape& s) {  // heads of a workgroup
  const int G = s.Hq / s.Hkv, fit = kTile / s.L;
  return fit < G ? fit : G;
}
__host__ __device__ inline int sp_groups(const Shape& s) {  // workgroups of a range and KV head
  const int G = s.Hq / s.Hkv;
  return (G + sp_pack(s) - 1) / sp_pack(s);
}
template <int D>
__global__ __launch_bounds__(kWave * 4) void hyb_sp_token_kernel(SoftmaxPrefixArgs a, SpCut cut) {
  typedef SpAcc<D> A;
  typedef RowColTile<D> RT;
  constexpr int NCT = A::NCT, NW = 4;
  struct alignas(16) Slot {
    bf16 k[kTile * D], v[kTile * D];
  };
  __shared__ Slot ring[NW][2];
  __shared__ float refs[NW][kTile], sums[NW][kTile];
  __shared__ int pages[kMaxRangePages];

  const int lane = threadIdx.x & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L, G = Hq / Hkv, pack = sp_pack(a.s), groups = sp_groups(a.s);
  int at, hg;
  sp_place(groups, at, hg);
  const int g = at % Hkv, r = at / Hkv;
  static_assert(sizeof(ring) >= kPlanInts * sizeof(int), "the plan's scratch fits the slots");
  const SpRange rg = sp_range<true>(a, sp_plan<true>(a, cut, reinterpret_cast<int*>(&ring)), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int Lb = sp_block<true>(a, rg.b);
  // this lane's column: query i of head h
  const int i = li % L, hl = hg * pack + li / L, h = g * G + hl;
  const bool col = li < pack * L && hl < G && i < Lb;
  bf16x8 qop[A::KD];
  {
    const bf16* row = (const bf16*)a.q + (((size_t)rg.b * L + (col ? i : 0)) * Hq + (col ? h : g * G)) * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < A::KD; ++ks) qop[ks] = keep_if<bf16>(col, load_op<bf16>(row + ks * 16));
  }
  const SpTiles<D> t(a, rg, g, sp_keys<true>(a, rg.b) - Lb, pages);
  const RT rt(lane);
  const int mine = (rg.nt - w + NW - 1) / NW;  // this wave's tiles
  auto issue = [&](int n, Slot& s) __attribute__((always_inline)) {
    if (n >= mine) return;
    const int j0 = t.first_key(w + NW * n);
    t.template copy<RT::IK>(0, j0, 0, s.k, lane);
    t.template copy<RT::IK>(1, j0, 0, s.v, lane);
  };
  const float scale = kLog2e / sqrtf((float)D);
  A acc;
  auto step = [&](int n, Slot& s) __attribute__((always_inline)) {
    if (n + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * RT::IK) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    acc.add(t, rt, t.first_key(w + NW * n), s.k, s.v, qop, scale, hh);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read
    issue(n + 2, s);
  };
  issue(0, ring[w][0]);
  issue(1, ring[w][1]);
  for (int n = 0; n < mine; n += 2) {
    step(n, ring[w][0]);
    if (n + 1 < mine) step(n + 1, ring[w][1]);
  }

  // The waves' sums over one reference: wave w scales its own and leaves them in
  // LDS, then joins entries 32 w .. + 31 of every query.
  mma_settle<bf16>();
  const float l = acc.l + xor32(acc.l);
  if (hh == 0) refs[w][li] = acc.m;
  lds_barrier();  // (and the slots are free)
  float mm = refs[0][li];
#pragma unroll
  for (int x = 1; x < NW; ++x) mm = fmaxf(mm, refs[x][li]);
  const float f = __builtin_amdgcn_exp2f(acc.m - mm);
  if (hh == 0) sums[w][li] = l * f;
  f32x4* const parts = reinterpret_cast<f32x4*>(&ring);  // [wave][ct * 4 + e][lane]
  static_assert(sizeof(ring) >= NW * NCT * 4 * kWave * sizeof(f32x4), "the sums fit the slots");
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      parts[(w * NCT * 4 + ct * 4 + e) * kWave + lane] = f32x4{acc.acc[ct][4 * e] * f, acc.acc[ct][4 * e + 1] * f,
                                                                acc.acc[ct][4 * e + 2] * f, acc.acc[ct][4 * e + 3] * f};
  lds_barrier();
  if (w >= NCT || !col) return;
  float den = 0.0f;
#pragma unroll
  for (int x = 0; x < NW; ++x) den += sums[x][li];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f32x4 o = {};
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const f32x4 y = parts[(x * NCT * 4 + w * 4 + e) * kWave + lane];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += y[k];
    }
    sp_put<bf16, D>(a, rg, r, h, i, w * kTile + row_of(4 * e, hh), o, den);
  }
  if (w == 0 && hh == 0) sp_put_sum<D>(a, rg, r, h, i, mm, den);
}

// Blocks (2 or 4 query heads per KV head): a wave per head, as in the ring kernel,
// in two halves that take the range's tiles in turn and join their sums in LDS.
// A window's ranges are short, so what a call waits for is the steps of one, and
// the partial results of several per request cost as much as they save; so a
// workgroup takes a range in half the steps instead of a range half as long:
// 32 requests of 32 queries, window 512, 28.5 us by the ring kernel in ranges of 512
// keys, 22 so; 24 of a window of 1024 33 and 30.  What bounds it is the copies in
// flight (96 KiB per workgroup, about 3 us), where the workgroups are few.
template <int D, int NG>
__global__ __launch_bounds__(kWave * 2 * NG, 2) void hyb_sp_block_kernel(SoftmaxPrefixArgs a, SpCut cut) {
  typedef SpAcc<D> A;
  typedef RowColTile<D> RT;
  constexpr int NCT = A::NCT, R = 4;
  constexpr int IPW = 2 * RT::IK / NG;  // copies per wave and step: the half's first waves K's, the others V's
  static_assert(IPW * NG == 2 * RT::IK && 3 * IPW <= 63, "copies split evenly, and those in flight fit vmcnt");
  struct alignas(16) Slot {
    bf16 k[kTile * D], v[kTile * D];
  };
  __shared__ Slot ring[2][R];
  __shared__ float refs[2][NG][kTile], sums[2][NG][kTile];
  __shared__ int pages[kMaxRangePages];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = wave / NG, w = wave % NG;
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, L = a.s.L;
  const int g = blockIdx.x % Hkv, r = blockIdx.x / Hkv, h = g * NG + w;
  static_assert(sizeof(ring) >= kPlanInts * sizeof(int), "the plan's scratch fits the slots");
  const SpRange rg = sp_range<true>(a, sp_plan<true>(a, cut, reinterpret_cast<int*>(&ring)), r, lane);
  if (rg.b < 0) return;  // uniform: past the plan's last range
  const int Lb = sp_block<true>(a, rg.b);
  bf16x8 qop[A::KD];
  {
    const bf16* row = (const bf16*)a.q + (((size_t)rg.b * L + min(li, Lb - 1)) * Hq + h) * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < A::KD; ++ks) qop[ks] = keep_if<bf16>(li < Lb, load_op<bf16>(row + ks * 16));
  }
  const SpTiles<D> t(a, rg, g, sp_keys<true>(a, rg.b) - Lb, pages);
  const RT rt(lane);
  const int nsteps = (rg.nt + 1) / 2, mine = (rg.nt + 1 - half) / 2;
  const int kv = w * IPW / RT::IK, u0 = w * IPW % RT::IK;
  auto issue = [&](int n, Slot& s) __attribute__((always_inline)) {
    if (n < mine) t.template copy<IPW>(kv, t.first_key(half + 2 * n), u0, kv == 0 ? s.k : s.v, lane);
  };
  const float scale = kLog2e / sqrtf((float)D);
  A acc;
  // Tile n + 3 of the half goes to the slot of tile n - 1.
  auto step = [&](int n, auto S) __attribute__((always_inline)) {
    constexpr int SV = decltype(S)::value;
    const int later = mine - 1 - n;
    if (later >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * IPW) : "memory");
    else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPW) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier_nodrain();
    issue(n + 3, ring[half][(SV + 3) % R]);
    if (n < mine) acc.add(t, rt, t.first_key(half + 2 * n), ring[half][SV].k, ring[half][SV].v, qop, scale, hh);
  };
  issue(0, ring[half][0]);
  issue(1, ring[half][1]);
  issue(2, ring[half][2]);
  for (int n = 0; n < nsteps; n += R) {
    step(n, std::integral_constant<int, 0>{});
    if (n + 1 < nsteps) step(n + 1, std::integral_constant<int, 1>{});
    if (n + 2 < nsteps) step(n + 2, std::integral_constant<int, 2>{});
    if (n + 3 < nsteps) step(n + 3, std::integral_constant<int, 3>{});
  }

  // The halves' sums over one reference: each hands over half of the entries
  // and joins the others.
  mma_settle<bf16>();
  const float l = acc.l + xor32(acc.l);
  if (hh == 0) refs[half][w][li] = acc.m;
  lds_barrier_nodrain();  // (and the slots are free)
  const float mm = fmaxf(refs[0][w][li], refs[1][w][li]);
  const float f = __builtin_amdgcn_exp2f(acc.m - mm);
  if (hh == 0) sums[half][w][li] = l * f;
  constexpr int NH = NCT / 2;  // groups of 32 entries per half
  f32x4* const parts = reinterpret_cast<f32x4*>(&ring);  // [for half][w][ct * 4 + e][lane]
  static_assert(sizeof(ring) >= 2 * NG * NH * 4 * kWave * sizeof(f32x4), "the sums fit the slots");
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 y = {acc.acc[ct][4 * e] * f, acc.acc[ct][4 * e + 1] * f, acc.acc[ct][4 * e + 2] * f,
                       acc.acc[ct][4 * e + 3] * f};
      if (ct / NH != half) parts[((ct / NH * NG + w) * NH * 4 + ct % NH * 4 + e) * kWave + lane] = y;
    }
  lds_barrier_nodrain();
  if (li >= Lb) return;
  const float den = sums[0][w][li] + sums[1][w][li];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
    if (ct / NH == half)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f32x4 o = parts[((half * NG + w) * NH * 4 + ct % NH * 4 + e) * kWave + lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += acc.acc[ct][4 * e + k] * f;
        sp_put<bf16, D>(a, rg, r, h, li, ct * kTile + row_of(4 * e, hh), o, den);
      }
  if (half == 0 && hh == 0) sp_put_sum<D>(a, rg, r, h, li, mm, den);
}

// Ranges per request on average at most (the workspace and the grid hold
// that many): about 2048 workgroups of ranges of at least 512 keys.
int softmax_prefix_splits(const Shape& s, int max_prefix) {
  const long units = (long)s.B * s.Hkv;
  long want = units > 0 ? (2048 + units - 1) / units : 1;
  const long cap = ((long)max_prefix + s.L + 511) / 512;
  if (want > cap) want = cap;
  // no range longer than kMaxRange keys (the paged kernel stages a range's
  // page numbers in LDS)
  const long least = ((long)max_prefix + s.L + kMaxRange - 1) / kMaxRange;
  if (want < least) want = least;
  if (want < 1) want = 1;
  return (int)want;
}

// A window's kernels (bf16).  The token kernel where all heads of a KV head share a
// workgroup, or where its workgroups, one per group of heads, are at most 256 (a
// group reads every tile again; 8 requests of 32 queries, window 1024, 28 us by
// the block kernel); the block kernel while a request is one range of it.
static bool sp_tokens(const Shape& s) {
  return s.dtype == 1 && (sp_groups(s) == 1 || (long)s.B * s.Hkv * sp_groups(s) <= 256);
}
static bool sp_blocks(const Shape& s, int max_seen) {
  const int G = s.Hq / s.Hkv;
  return s.dtype == 1 && !sp_tokens(s) && (G == 2 || G == 4) && max_seen + s.L <= 2048;
}
// Ranges per request: one by the block kernel, and by the token kernel where
// its workgroups fill the chip anyway (a merge costs more than an even cut
// saves).
int softmax_window_splits(const Shape& s, int max_seen) {
  if (sp_blocks(s, max_seen)) return 1;
  const int n = softmax_prefix_splits(s, max_seen);
  if (!sp_tokens(s) || (long)max_seen + s.L > kMaxRange) return n;
  if ((long)s.B * s.Hkv * sp_groups(s) >= 256) return 1;
  // (ranges of 1024 keys and more where the heads have workgroups of their own)
  return sp_groups(s) == 1 ? n : std::max(1, std::min(n, (int)(((long)max_seen + s.L) / 1024)));
}

// A single KV range per (request, KV head) writes the normalised output
// directly and needs no workspace.
size_t softmax_prefix_ws_bytes(const Shape& s, int n_split) {
  if (n_split <= 1) return 0;
  return (size_t)s.B * s.Hq * n_split * s.L * (s.D + 2) * sizeof(float);
}

template <typename T, int D, bool PAGED, bool WIN>
static hipError_t sp_go(const SoftmaxPrefixArgs& a, hipStream_t st) {
  SpCut cut;
  hipError_t e;
  // (a paged cache is cut as the contiguous one is, for the same bits: by what fits
  // of both their kernels)
#define HYB_SP_CASE(NG, RING, ...)                                              \
  case NG: {                                                                    \
    static const int resident =                                                 \
        WIN ? sp_resident(__VA_ARGS__, true, true>, NG)                         \
            : min(sp_resident(__VA_ARGS__, true>, NG), sp_resident(__VA_ARGS__, false>, NG)); \
    e = sp_launch(__VA_ARGS__, PAGED, WIN>, resident, NG, RING, a, st, &cut);   \
    break;                                                                      \
  }
  // bf16 with 1, 2, 4 or 8 query heads per KV head: the copy ring; else the
  // register-staged kernel.
  if (WIN && sp_tokens(a.s)) {
    static const int resident = sp_resident(hyb_sp_token_kernel<D>, 4);
    e = sp_launch(hyb_sp_token_kernel<D>, resident, 4, true, a, st, &cut, sp_groups(a.s));
  } else if (WIN && sp_blocks(a.s, a.max_seen) && a.s.Hq / a.s.Hkv == 2) {
    static const int resident = sp_resident(hyb_sp_block_kernel<D, 2>, 4);
    e = sp_launch(hyb_sp_block_kernel<D, 2>, resident, 4, true, a, st, &cut);
  } else if (WIN && sp_blocks(a.s, a.max_seen)) {
    static const int resident = sp_resident(hyb_sp_block_kernel<D, 4>, 8);
    e = sp_launch(hyb_sp_block_kernel<D, 4>, resident, 8, true, a, st, &cut);
  } else if constexpr (sizeof(T) == 2) {
    switch (a.s.Hq / a.s.Hkv) {
      HYB_SP_CASE(2, true, hyb_sp_ring_kernel<D, 2)
      HYB_SP_CASE(3, false, hyb_sp_partial_kernel<T, D, 3)
      HYB_SP_CASE(4, true, hyb_sp_ring_kernel<D, 4)
      HYB_SP_CASE(5, false, hyb_sp_partial_kernel<T, D, 5)
      HYB_SP_CASE(6, false, hyb_sp_partial_kernel<T, D, 6)
      HYB_SP_CASE(7, false, hyb_sp_partial_kernel<T, D, 7)
      HYB_SP_CASE(8, true, hyb_sp_ring_kernel<D, 8)
      default:
        if constexpr (!WIN) {  // (a window's single head takes the token kernel)
          switch (a.s.Hq / a.s.Hkv) {
            HYB_SP_CASE(1, true, hyb_sp_ring_kernel<D, 1)
            default: return hipErrorInvalidValue;
          }
          break;
        }
        return hipErrorInvalidValue;
    }
  } else {
    switch (a.s.Hq / a.s.Hkv) {
      HYB_SP_CASE(1, false, hyb_sp_partial_kernel<T, D, 1)
      HYB_SP_CASE(2, false, hyb_sp_partial_kernel<T, D, 2)
      HYB_SP_CASE(3, false, hyb_sp_partial_kernel<T, D, 3)
      HYB_SP_CASE(4, false, hyb_sp_partial_kernel<T, D, 4)
      HYB_SP_CASE(5, false, hyb_sp_partial_kernel<T, D, 5)
      HYB_SP_CASE(6, false, hyb_sp_partial_kernel<T, D, 6)
      HYB_SP_CASE(7, false, hyb_sp_partial_kernel<T, D, 7)
      HYB_SP_CASE(8, false, hyb_sp_partial_kernel<T, D, 8)
      default: return hipErrorInvalidValue;
    }
  }
#undef HYB_SP_CASE
  if (e != hipSuccess || a.n_split == 1) return e;  // one range: already written out
  const long units = (long)a.s.B * a.s.Hq * ((a.s.L + 1024 / D - 1) / (1024 / D));
  hipLaunchKernelGGL((hyb_sp_combine_kernel<T, D, WIN>), dim3((unsigned)std::min<long>(units, 2048)), dim3(256), 0, st,
                     a, cut);
  return hipGetLastError();
}

template <bool PAGED, bool WIN = false>
static hipError_t sp_dispatch(const SoftmaxPrefixArgs& a, hipStream_t st) {
  if (a.s.dtype == 1)
    return a.s.D == 64 ? sp_go<bf16, 64, PAGED, WIN>(a, st) : sp_go<bf16, 128, PAGED, WIN>(a, st);
  return a.s.D == 64 ? sp_go<float, 64, PAGED, WIN>(a, st) : sp_go<float, 128, PAGED, WIN>(a, st);
}

hipError_t launch_softmax_prefix(const SoftmaxPrefixArgs& a, hipStream_t st) {
  if (a.s.Hq / a.s.Hkv > kMaxGroup) return hipErrorInvalidValue;
  // (without pages no token is cached: max_prefix is 0 and the pools are not read)
  if (a.window >= 0) return sp_dispatch<true, true>(a, st);
  if (a.page_table) {
    if (a.page_shift < 5 || a.n_pages < 1) return hipErrorInvalidValue;
    return sp_dispatch<true>(a, st);
  }
  return sp_dispatch<false>(a, st);
}

}  // namespace hyb
