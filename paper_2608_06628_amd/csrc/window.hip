// window.hip -- softmax attention over a sequence in which a token sees its
// own block, the `window` tokens before the block and the first n_sinks
// tokens, and its gradient: the block-causal pattern of Figure 2 with the
// softmax of Section 2.2 in place of the state, as the softmax layers that
// stay beside the hybrid ones run it over a prompt, as the teacher of the
// attention transfer runs it (window >= T: every earlier block), and as their
// end-to-end training differentiates it.
//
// For query i with block start s = (i / L) L:
//   seen(i) = { j < min(s + L, len) : j >= s - window or j < n_sinks }
//   out_i = sum_j P_ij v_j,  P_ij = exp(q_i k_j / sqrt(d) - lse_i)
//   dP_ij = dout_i v_j,  dS_ij = P_ij (dP_ij - delta_i),  delta_i = dout_i out_i
//   dv_j = sum_i P_ij dout_i,  dq_i = sum_j dS_ij k_j / sqrt(d),
//   dk_j = sum_i dS_ij q_i / sqrt(d)
// A query always sees itself, so no row is empty.
//
// Bound: the matrix cores (4 d flops per pair of query and key forward, 14 d
// backward, where the scores and dP are formed by both gradient kernels so
// that each gradient is summed by the wave that owns its rows: no atomics,
// the same bits every time).  Products are 32x32 tiles, transposed so that
// each accumulator tile is the next product's operand without leaving its
// registers (device.h).
//
// Measured, bf16, 16 and 4 heads of d = 128, calls one after the other: 8 x 8192 tokens, window
// 4096, 1.67 to 1.78 ms (940 to 1000 TFLOP/s; a product of 8192 cubed reaches 1180 to 1210 on the
// same cards, and the clock falls to 1.85 GHz for both); gradient of 8 x 2048 tokens, every earlier
// block, 480 to 513 us (0.68 to 0.73 PFLOP/s of 10 d per pair).
//
// Packed sequences (PackedArgs) go through the same kernels: a workgroup finds its sequence, and
// its place there, from the starts on the device (ragged.h; 2 to 7% of a call for equal
// lengths beside the padded one).  24 sequences of 170 to 4096 tokens, blocks of 32, every earlier
// block, 710 us (800 TFLOP/s); gradient of 16 of 128 to 2048, causal, 410 to 418 us; of 40 of 13 to 511, window 255, 8
// and 2 heads of d = 64, 54 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device.h"
#include "launch.h"
#include "launch_packed.h"
#include "ragged.h"

namespace hyb {

// Reference of a query that has seen no key yet: finite, so that a tile in
// which it sees none leaves weights of exactly zero.
constexpr float kNoRef = -1e30f;

// What query i (below len) sees: keys lo .. end - 1, and those below sinks.
struct WinRow {
  int lo, end;
  __device__ inline WinRow(const WindowArgs& a, int len, int i) {
    const int s0 = i / a.s.L * a.s.L;
    lo = max(0, s0 - a.window);
    end = min(s0 + min(a.s.L, len - s0), len);
  }
  __device__ inline bool sees(int j, int sinks) const { return (j < end) & ((j >= lo) | (j < sinks)); }
};

// The key tiles that the queries i0 .. i1 - 1 see some of: tiles 0 .. st - 1
// (the sinks) and from st + skip on, n in all.
struct WinTiles {
  int st, skip, n;
  __device__ inline WinTiles(const WindowArgs& a, int len, int i0, int i1, int tile) {
    const int lo = WinRow(a, len, i0).lo, end = WinRow(a, len, i1 - 1).end;
    st = (min(a.n_sinks, lo) + tile - 1) / tile;
    skip = max(0, lo / tile - st);
    n = (end + tile - 1) / tile - skip;
  }
  __device__ inline int first(int x, int tile) const { return (x < st ? x : x + skip) * tile; }
};

// Queries i0 .. i1 - 1 and the keys j0 .. j0 + n - 1: whether every query sees
// every key, and whether any sees any.
__device__ inline bool win_full(const WinRow& r0, const WinRow& r1, int sinks, int j0, int n) {
  return j0 + n <= r0.end && (j0 >= r1.lo || j0 + n <= sinks);
}
__device__ inline bool win_none(const WinRow& r0, const WinRow& r1, int sinks, int j0, int n) {
  return j0 >= r1.end || (j0 + n <= r0.lo && j0 >= sinks);
}

// The keys' side of WinRow: key j is seen by the queries q0 .. q1 - 1.
struct WinKey {
  int q0, q1;
  __device__ inline WinKey(const WindowArgs& a, int len, int j) {
    const int L = a.s.L;
    q0 = j / L * L;
    const long end = ((long)j + a.window) / L * L + L;
    q1 = j < a.n_sinks ? len : (int)min(end, (long)len);
  }
};

// The workgroups' order: the x-th workgroups of all (request, KV head)s one after
// the other, so that with the longest first the chip ends with short ones; a
// (request, KV head) stays on one XCD where their number is a multiple of 8
// (workgroups go to the XCDs in turn), which keeps what it reads in that XCD's L2.
// (One (request, KV head) after the other left the last one's long workgroups
// to the end: gradient of 8 x 2048 tokens 618 us, now 503.)
__device__ inline void win_place(int bid, int nbg, int& bg, int& x) {
  bg = bid % nbg;
  x = bid / nbg;
}

// Units of the query kernels (32 queries of a head) per workgroup, at most; keys of a
// workgroup of the dK, dV kernels.
constexpr int kWinWaves = 4;
constexpr int kWinKeys = 4 * kTile;

// A sequence: its tokens, the rows that are its own (those past its tokens get gradients
// of zero), and where they are.  Offsets are of a head's entries of its first row.
template <typename A>
struct WinSeq;
template <>
struct WinSeq<WindowArgs> {
  const WindowArgs& a;
  int b, len, cap;
  __device__ inline WinSeq(const WindowArgs& a_, int b_)
      : a(a_), b(b_), len(a_.seq_lens ? min(max(a_.seq_lens[b_], 0), a_.T) : a_.T), cap(a_.T) {}
  __device__ inline size_t q(int h, int D) const { return ((size_t)b * a.T * a.s.Hq + h) * D; }
  __device__ inline size_t k(int g, int D) const { return ((size_t)b * a.T * a.s.Hkv + g) * D; }
  __device__ inline size_t v(int g, int D) const { return k(g, D); }
  __device__ inline size_t dout(int h, int D) const { return q(h, D); }
  // from a row to the next
  __device__ inline size_t qs(int D) const { return (size_t)a.s.Hq * D; }
  __device__ inline size_t ks(int D) const { return (size_t)a.s.Hkv * D; }
  __device__ inline size_t vs(int D) const { return ks(D); }
  __device__ inline size_t row(int i) const { return (size_t)b * a.T + i; }         // of out, the gradients
  __device__ inline size_t lse(int h, int i) const { return ((size_t)b * a.s.Hq + h) * a.T + i; }
  // of the bf16 gradient's statistics: [B][Hq][Tp], Tp = T rounded up to a tile
  __device__ inline size_t stats(int h, int i) const { return ((size_t)b * a.s.Hq + h) * ((a.T + kTile - 1) / kTile * kTile) + i; }
};
// Packed: one sequence more than there are, of no tokens, has the rows behind the last.
__host__ __device__ inline long win_packed_tiles(int start, int b) { return (long)(start / kTile) + b; }
template <>
struct WinSeq<PackedArgs> {
  const PackedArgs& a;
  int b, len, cap, start;
  __device__ inline WinSeq(const PackedArgs& a_, int b_) : a(a_), b(b_) {
    start = ragged_start(a.token_start, b, a.N);
    len = b < a.s.B ? max(ragged_start(a.token_start, b + 1, a.N) - start, 0) : 0;
    cap = b < a.s.B ? len : a.N - start;
  }
  __device__ inline size_t q(int h, int D) const { return (size_t)start * a.q_stride + (size_t)h * D; }
  __device__ inline size_t k(int g, int D) const { return (size_t)start * a.k_stride + (size_t)g * D; }
  __device__ inline size_t v(int g, int D) const { return (size_t)start * a.v_stride + (size_t)g * D; }
  __device__ inline size_t dout(int h, int D) const { return ((size_t)start * a.s.Hq + h) * D; }
  __device__ inline size_t qs(int) const { return a.q_stride; }
  __device__ inline size_t ks(int) const { return a.k_stride; }
  __device__ inline size_t vs(int) const { return a.v_stride; }
  __device__ inline size_t row(int i) const { return (size_t)start + i; }
  __device__ inline size_t lse(int h, int i) const { return (size_t)h * a.N + start + i; }
  // [Hq][tiles of all sequences][32]
  __device__ inline size_t stats(int h, int i) const {
    return ((size_t)h * win_packed_tiles(a.N, a.s.B + 1) + win_packed_tiles(start, b)) * kTile + i;
  }
};

// Packed: the first workgroup of the queries of sequence b, and of its keys, so that
// every sequence has room for its own: of U units, G per tile of queries, and of 128 keys.
__host__ __device__ inline long win_packed_queries(int start, int b, int G, int U = kWinWaves) {
  return (long)start * G / (U * kTile) + (long)b * ((G + U - 1) / U + 2);
}
__host__ __device__ inline long win_packed_keys(int start, int b) { return (long)(start / kWinKeys) + b; }

// This workgroup's sequence, KV head, and its place x among the sequence's
// workgroups of queries, of `wgs` (per sequence and head, or packed per head); those of the
// last queries, which see most, come first.
template <int U = kWinWaves>
__device__ inline WinSeq<WindowArgs> win_of_queries(const WindowArgs& a, int wgs, int, int& g, int& x) {
  int bg;
  win_place(blockIdx.x, a.s.B * a.s.Hkv, bg, x);
  x = wgs - 1 - x;
  g = bg % a.s.Hkv;
  return WinSeq<WindowArgs>(a, bg / a.s.Hkv);
}
template <int U = kWinWaves>
__device__ inline WinSeq<PackedArgs> win_of_queries(const PackedArgs& a, int wgs, int lane, int& g, int& x) {
  const int G = a.s.Hq / a.s.Hkv;
  win_place(blockIdx.x, a.s.Hkv, g, x);
  if (a.s.B < kMaxLevelled) {  // the longest lists first, of all sequences
    int level = 0;
    const int b = ragged_level(a.s.B + 1, x, lane, [&](int i) {
      return ((WinSeq<PackedArgs>(a, i).cap + kTile - 1) / kTile * G + U - 1) / U;
    }, level);
    WinSeq<PackedArgs> s(a, max(b, 0));
    if (b < 0) s.len = s.cap = 0;
    x = level;
    return s;
  }
  x = wgs - 1 - x;
  const int b = ragged_find(a.s.B + 1, x, lane,
                            [&](int i) { return win_packed_queries(ragged_start(a.token_start, i, a.N), i, G, U); });
  const WinSeq<PackedArgs> s(a, b);
  x = max(0, x - (int)win_packed_queries(s.start, b, G, U));
  return s;
}

// The dK, dV kernels: a workgroup owns 128 keys and goes through the query
// tiles that see them, of all heads of the KV head.  These lists are cut into
// parts that are summed in the workspace: those of the keys among the sinks, which
// every later query sees (the first `ns` workgroups of a (request, KV head)), into
// ps, the others into p.
struct WinParts {
  int wgs, ns, ps, p;
  bool halves;  // (bf16) workgroups of two halves
  __host__ __device__ int items() const { return ns * ps + (wgs - ns) * p; }
  // Rows of partial sums of dK and dV: ps for the first ns workgroups' keys
  // (padded), then p of every key, each where there is more than one.
  __host__ __device__ long sink_rows() const { return ps > 1 ? (long)ps * ns * kWinKeys : 0; }
  __host__ __device__ long rows(int T) const { return sink_rows() + (p > 1 ? (long)p * T : 0); }
};
// Item y of a (request, KV head): its keys' workgroup x and part; and where its
// results go: key j's row of dK (o = 0) or dV (o = 1) in the sums
// [part][o][B][span][Hkv][D] of its region.
struct WinItem {
  int x, part, parts, span;
  bool sink;
  __device__ inline WinItem() {}
  __device__ inline WinItem(const WindowArgs& a, const WinParts& c, int y) {
    sink = y < c.ns * c.ps;
    parts = sink ? c.ps : c.p;
    if (!sink) y -= c.ns * c.ps;
    part = y % parts;
    x = y / parts + (sink ? 0 : c.ns);
    span = sink ? c.ns * kWinKeys : a.T;
  }
  template <int D>
  __device__ inline float* sums(const WindowArgs& a, const WinParts& c) const {
    return a.sums + (sink ? 0 : c.sink_rows() * 2 * a.s.B * a.s.Hkv * D);
  }
  __device__ inline size_t row(const WinSeq<WindowArgs>& s, int o, int j, int g) const {
    return (((size_t)(part * 2 + o) * s.a.s.B + s.b) * span + j) * s.a.s.Hkv + g;
  }
  __device__ inline size_t row(const WinSeq<PackedArgs>& s, int o, int j, int g) const {
    return ((size_t)(part * 2 + o) * s.a.N + s.row(j)) * s.a.s.Hkv + g;
  }
};
// This workgroup's sequence, KV head and item; those of the first keys, which most queries
// see, come first.  Packed: every list has p parts, also the sinks', with the sums
// [part][o][N][Hkv][D].
__device__ inline WinSeq<WindowArgs> win_of_keys(const WindowArgs& a, const WinParts& cut, int, int& g, WinItem& it) {
  int bg, y;
  win_place(blockIdx.x, a.s.B * a.s.Hkv, bg, y);
  it = WinItem(a, cut, y);
  g = bg % a.s.Hkv;
  return WinSeq<WindowArgs>(a, bg / a.s.Hkv);
}
__device__ inline WinSeq<PackedArgs> win_of_keys(const PackedArgs& a, const WinParts& cut, int lane, int& g, WinItem& it) {
  int y;
  win_place(blockIdx.x, a.s.Hkv, g, y);
  it.sink = false;
  it.parts = cut.p;
  it.part = y % cut.p;
  const int x = y / cut.p;
  if (a.s.B < kMaxLevelled) {
    auto count = [&](int i) { return (WinSeq<PackedArgs>(a, i).cap + kWinKeys - 1) / kWinKeys; };
    int level = 0;
    const int b = ragged_level(a.s.B + 1, x, lane, count, level);
    WinSeq<PackedArgs> s(a, max(b, 0));
    it.x = (s.cap + kWinKeys - 1) / kWinKeys - 1 - level;
    if (b < 0) s.len = s.cap = it.x = 0;
    return s;
  }
  const int b = ragged_find(a.s.B + 1, x, lane,
                            [&](int i) { return win_packed_keys(ragged_start(a.token_start, i, a.N), i); });
  const WinSeq<PackedArgs> s(a, b);
  it.x = max(0, x - (int)win_packed_keys(s.start, b));
  return s;
}

// ---- fp32 kernels -------------------------------------------------------------
//
// One wave per 32 rows (queries of a head; keys of a KV head in the dK, dV
// kernel), four waves per workgroup sharing the pairs of tiles they loop over
// through LDS: the next pair is in registers on its way from memory while this
// one is used, and moves to the other buffer at the end of the step, so a step has
// one barrier.  fp32 products run at 1/16 of the bf16 rate and bound the loop (a
// pair of tiles at d = 64 is 128 products of 64 cycles for the four waves' SIMDs).

template <int D, int W = kWinWaves>  // W: waves that share a tile's copies
struct WinF32 {
  typedef Mma<float> M;
  static constexpr int KD = D / M::KW, NCT = D / kTile;
  static constexpr int LD = D + 4;             // row pitch in LDS
  static constexpr int NCH = kTile * D / 4 / (kWave * W);  // 16-byte pieces of a tile per thread
  typedef float Tile[kTile][LD];
  typedef float Ops[KD];
  typedef f32x16 Acc[NCT];
  struct Regs {
    f32x4 a[NCH], b[NCH];
  };
};

// Rows row0 .. row0 + 31 of two arrays (row strides in elements) into registers,
// and from there, zero from row `rows` on, into two tiles; by W waves, whose
// thread number t is.  (The zeros are put in last: a select at the load would wait for it.)
template <int D, int W = kWinWaves>
__device__ inline void win_fetch(typename WinF32<D, W>::Regs& r, const float* a, const float* b, size_t as,
                                 size_t bs, int row0, int rows, int t) {
#pragma unroll
  for (int u = 0; u < WinF32<D, W>::NCH; ++u) {
    const int x = t + u * kWave * W, i = row0 + x / (D / 4);
    const int row = min(i, rows - 1), c = x % (D / 4) * 4;
    r.a[u] = *reinterpret_cast<const f32x4*>(a + row * as + c);
    r.b[u] = *reinterpret_cast<const f32x4*>(b + row * bs + c);
  }
}
template <int D, int W = kWinWaves>
__device__ inline void win_put(const typename WinF32<D, W>::Regs& r, typename WinF32<D>::Tile& a,
                               typename WinF32<D>::Tile& b, int row0, int rows, int t) {
#pragma unroll
  for (int u = 0; u < WinF32<D, W>::NCH; ++u) {
    const int x = t + u * kWave * W, i = x / (D / 4);
    const bool ok = row0 + i < rows;
    *reinterpret_cast<f32x4*>(&a[i][x % (D / 4) * 4]) = ok ? r.a[u] : f32x4{};
    *reinterpret_cast<f32x4*>(&b[i][x % (D / 4) * 4]) = ok ? r.b[u] : f32x4{};
  }
}
// The entry of a row that step ks of a product over d contracts in lane half
// hh: any order will do that both operands share, and this one makes four steps
// one 16-byte piece.
__device__ constexpr int win_entry(int ks, int hh) { return ks / 4 * 8 + 4 * hh + ks % 4; }
// A row as an operand (zero past the last row).
template <int D>
__device__ inline void win_row_ops(typename WinF32<D>::Ops& op, const float* row, bool ok, int hh) {
#pragma unroll
  for (int ks = 0; ks < WinF32<D>::KD; ks += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(row + win_entry(ks, hh));
#pragma unroll
    for (int k = 0; k < 4; ++k) op[ks + k] = ok ? v[k] : 0.0f;
  }
}
// tile rows times the operands of 32 columns: rows in accumulator order.
template <int D>
__device__ inline f32x16 win_rows_mma(const typename WinF32<D>::Tile& t, const float* op, int li, int hh) {
  f32x16 s = {};
#pragma unroll
  for (int ks = 0; ks < WinF32<D>::KD; ks += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(&t[li][win_entry(ks, hh)]);
#pragma unroll
    for (int k = 0; k < 4; ++k) s = Mma<float>::mma(v[k], op[ks + k], s);
  }
  mma_settle<float>();
  return s;
}
// acc[D][32] += tile^T x, x in accumulator order over the tile's rows.
template <int D>
__device__ inline void win_cols_mma(typename WinF32<D>::Acc& acc, const typename WinF32<D>::Tile& t, const float (&x)[16],
                                    int li, int hh) {
#pragma unroll
  for (int ct = 0; ct < WinF32<D>::NCT; ++ct)
#pragma unroll
    for (int ks = 0; ks < 16; ++ks) acc[ct] = Mma<float>::mma(t[row_of(ks, hh)][ct * kTile + li], x[ks], acc[ct]);
}
// acc^T (times f) to row `row` of out; entries CT0 * 32 .. CT1 * 32 - 1.
template <typename T, int D, int CT0 = 0, int CT1 = D / kTile>
__device__ inline void win_store(void* out, size_t row, const f32x16 (&acc)[D / kTile], float f, int hh, bool f32) {
#pragma unroll
  for (int ct = CT0; ct < CT1; ++ct)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float o[4] = {acc[ct][i] * f, acc[ct][i + 1] * f, acc[ct][i + 2] * f, acc[ct][i + 3] * f};
      store_out4<T>(out, row * D + ct * kTile + row_of(i, hh), o, f32);
    }
}

// Units of the query kernels: 32 queries of one head; the heads of a KV head
// vary fastest, so that a workgroup's waves share their keys.
struct WinUnit {
  int h, i0;  // query head, first query
  bool any;
};
__device__ inline WinUnit win_unit(const WindowArgs& a, int len, int g, int u) {
  const int G = a.s.Hq / a.s.Hkv;
  const int i0 = u / G * kTile;
  return WinUnit{g * G + u % G, i0, i0 < len};
}

// A wave's 32 queries take the keys j0 .. j0 + 31 (`full`, uniform: every query sees every one): m is the
// reference of the weights in the log2 domain, l their sum, acc the weighted sums of V^T.
template <int D>
__device__ __attribute__((always_inline)) inline void win_take(typename WinF32<D>::Acc& acc, float& m, float& l, const typename WinF32<D>::Tile& kt,
                                const typename WinF32<D>::Tile& vt, const float* qop, const WinRow& row, bool full,
                                int sinks, int j0, float scale, int li, int hh) {
  f32x16 sc = win_rows_mma<D>(kt, qop, li, hh);
  if (!full) {
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = row.sees(j0 + row_of(e, hh), sinks) ? sc[e] : -INFINITY;
  }
  float p[16], mt = sc[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
  mt = fmaxf(mt, xor32(mt)) * scale;
  const float mn = fmaxf(m, mt);
  if (__any(mn > m)) {
    mma_settle<float>();
    const float corr = __builtin_amdgcn_exp2f(m - mn);
    l *= corr;
#pragma unroll
    for (int ct = 0; ct < WinF32<D>::NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[ct][e] *= corr;
    m = mn;
  }
  float ps = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -m));
    ps += p[e];
  }
  l += ps + xor32(ps);
  win_cols_mma<D>(acc, vt, p, li, hh);
  mma_settle<float>();
}
// The same for dQ: weights from the rows' lse (log2), times dP - delta.
template <int D>
__device__ __attribute__((always_inline)) inline void win_take_dq(typename WinF32<D>::Acc& acc, const typename WinF32<D>::Tile& kt,
                                   const typename WinF32<D>::Tile& vt, const float* qop, const float* dop, const WinRow& row,
                                   bool full, int sinks, int j0, float scale, float lse, float delta, int li, int hh) {
  f32x16 sc = win_rows_mma<D>(kt, qop, li, hh);
  const f32x16 dp = win_rows_mma<D>(vt, dop, li, hh);
  if (!full) {
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = row.sees(j0 + row_of(e, hh), sinks) ? sc[e] : -INFINITY;
  }
  float ds[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -lse)) * (dp[e] - delta);
  win_cols_mma<D>(acc, kt, ds, li, hh);
  mma_settle<float>();
}

// Forward, of U units per workgroup.  With H = 2 two halves of U waves take a unit's tiles in turn, each
// through buffers of its own, and join their sums in LDS: a CU that holds one
// workgroup has two waves per SIMD then, and one's products run beside the other's
// weights (3 x 1197 tokens, 8 heads of d = 64, window 300: 47 us with one half, now 40).
template <int D, int H, typename A, int U = kWinWaves>
__global__ __launch_bounds__(kWave* U* H) void hyb_win_fwd_kernel(A a, int wgs) {
  typedef WinF32<D, U> C;
  struct Tiles {
    typename C::Tile k[H][2], v[H][2];
  };
  struct Join {  // the second half's sums and weighted sums
    float m[U][kTile], l[U][kTile];
    f32x4 x[U][C::NCT * 4][kWave];
  };
  union Smem {
    Tiles tiles;
    Join join;
    __device__ Smem() {}
  };
  __shared__ alignas(16) Smem sh;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = wave / U, w = wave % U, t = threadIdx.x % (kWave * U);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g, x;
  const WinSeq<A> sq = win_of_queries<U>(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x * U + w);
  const int first = x * U / G * kTile, last = min(((x + 1) * U - 1) / G * kTile + kTile, len);
  if (first >= len) return;  // uniform
  const WinTiles tl(a, len, first, last, kTile);
  const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
  const float* K = (const float*)a.k + sq.k(g, D);
  const float* V = (const float*)a.v + sq.v(g, D);
  const int i = min(me.i0 + li, len - 1);
  const WinRow row(a, len, i), r0(a, len, min(me.i0, len - 1)), r1(a, len, min(me.i0 + kTile, len) - 1);
  // This half's step n takes tile H n + half.
  typename C::Tile(&kt)[2] = sh.tiles.k[half];
  typename C::Tile(&vt)[2] = sh.tiles.v[half];
  const int nsteps = (tl.n + H - 1) / H, mine = (tl.n + H - 1 - half) / H;
  auto key = [&](int n) __attribute__((always_inline)) { return tl.first(H * n + half, kTile); };
  typename C::Regs next;
  if (mine > 0) win_fetch<D, U>(next, K, V, ks_, vs_, key(0), len, t);
  typename C::Ops qop;
  win_row_ops<D>(qop, (const float*)a.q + sq.q(me.h, D) + i * qs, true, hh);
  const float scale = kLog2e / sqrtf((float)D);
  float m = kNoRef, l = 0.0f;
  typename C::Acc acc;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) acc[ct] = f32x16{};
  if (mine > 0) win_put<D, U>(next, kt[0], vt[0], key(0), len, t);
  __syncthreads();
  for (int n = 0; n < nsteps; ++n) {
    const int buf = n & 1, j0 = n < mine ? key(n) : 0;
    if (n + 1 < mine) win_fetch<D, U>(next, K, V, ks_, vs_, key(n + 1), len, t);
    if (me.any && n < mine && !win_none(r0, r1, a.n_sinks, j0, kTile))  // uniform over the wave
      win_take<D>(acc, m, l, kt[buf], vt[buf], qop, row, win_full(r0, r1, a.n_sinks, j0, kTile), a.n_sinks, j0, scale, li, hh);
    if (n + 1 < mine) win_put<D, U>(next, kt[buf ^ 1], vt[buf ^ 1], key(n + 1), len, t);
    __syncthreads();
  }
  if constexpr (H == 2) {
    if (half == 1) {
      if (hh == 0) {
        sh.join.m[w][li] = m;
        sh.join.l[w][li] = l;
      }
#pragma unroll
      for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sh.join.x[w][ct * 4 + e][lane] =
              f32x4{acc[ct][4 * e], acc[ct][4 * e + 1], acc[ct][4 * e + 2], acc[ct][4 * e + 3]};
    }
    __syncthreads();
    if (half == 1) return;
    const float mo = sh.join.m[w][li], mm = fmaxf(m, mo);
    const float f = __builtin_amdgcn_exp2f(m - mm), fo = __builtin_amdgcn_exp2f(mo - mm);
    l = l * f + sh.join.l[w][li] * fo;
    m = mm;
#pragma unroll
    for (int ct = 0; ct < C::NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 y = sh.join.x[w][ct * 4 + e][lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[ct][4 * e + k] = acc[ct][4 * e + k] * f + y[k] * fo;
      }
  }
  if (!me.any || me.i0 + li >= len) return;
  win_store<float, D>(a.out, sq.row(i) * Hq + me.h, acc, 1.0f / l, hh, true);
  if (a.lse && hh == 0) a.lse[sq.lse(me.h, i)] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// dQ, and delta of the rows for the dK, dV kernel.
template <int D, typename A>
__global__ __launch_bounds__(kWave* kWinWaves) void hyb_win_dq_kernel(A a, int wgs) {
  typedef WinF32<D> C;
  __shared__ alignas(16) typename C::Tile kt[2], vt[2];
  const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g, x;
  const WinSeq<A> sq = win_of_queries(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x * kWinWaves + w);
  const int first = x * kWinWaves / G * kTile, last = min(((x + 1) * kWinWaves - 1) / G * kTile + kTile, len);
  const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
  typename C::Acc acc;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) acc[ct] = f32x16{};
  if (first < len) {  // uniform
    const WinTiles tl(a, len, first, last, kTile);
    const float* K = (const float*)a.k + sq.k(g, D);
    const float* V = (const float*)a.v + sq.v(g, D);
    const int i = min(me.i0 + li, len - 1);
    const WinRow row(a, len, i), r0(a, len, min(me.i0, len - 1)), r1(a, len, min(me.i0 + kTile, len) - 1);
    typename C::Regs next;
    win_fetch<D>(next, K, V, ks_, vs_, tl.first(0, kTile), len, threadIdx.x);
    typename C::Ops qop, dop;
    const size_t at = sq.dout(me.h, D) + (size_t)i * Hq * D;
    win_row_ops<D>(qop, (const float*)a.q + sq.q(me.h, D) + i * qs, true, hh);
    win_row_ops<D>(dop, (const float*)a.dout + at, true, hh);
    float delta = 0.0f;
#pragma unroll
    for (int ks = 0; ks < C::KD; ++ks) delta += dop[ks] * ((const float*)a.out)[at + win_entry(ks, hh)];
    delta += xor32(delta);
    const float scale = kLog2e / sqrtf((float)D);
    const size_t st = sq.lse(me.h, i);
    const float lse = a.lse[st] * kLog2e;
    if (hh == 0 && me.i0 + li < len) a.ws[st] = delta;
    win_put<D>(next, kt[0], vt[0], tl.first(0, kTile), len, threadIdx.x);
    __syncthreads();
    for (int n = 0; n < tl.n; ++n) {
      const int j0 = tl.first(n, kTile), buf = n & 1;
      if (n + 1 < tl.n) win_fetch<D>(next, K, V, ks_, vs_, tl.first(n + 1, kTile), len, threadIdx.x);
      if (me.any && !win_none(r0, r1, a.n_sinks, j0, kTile))
        win_take_dq<D>(acc, kt[buf], vt[buf], qop, dop, row, win_full(r0, r1, a.n_sinks, j0, kTile), a.n_sinks, j0, scale,
                       lse, delta, li, hh);
      if (n + 1 < tl.n) win_put<D>(next, kt[buf ^ 1], vt[buf ^ 1], tl.first(n + 1, kTile), len, threadIdx.x);
      __syncthreads();
    }
  }
  if (me.i0 + li >= sq.cap) return;  // rows past the length: zero
  win_store<float, D>(a.dq, sq.row(me.i0 + li) * Hq + me.h, acc,
                      me.i0 + li < len ? 1.0f / sqrtf((float)D) : 0.0f, hh, true);
}

// Few units: a workgroup per unit, whose waves take the unit's tiles in turn, each through a pair
// of tiles of its own (no barrier in the loop), and join their sums in LDS.
template <int D>
struct WinFew {
  typedef WinF32<D, 1> C;
  static constexpr int NW = kWinWaves, NCT = C::NCT;
  union {
    struct {
      typename C::Tile k[NW], v[NW];
    } tiles;
    f32x4 parts[NW][NCT * 4][kWave];
  };
  float m[NW][kTile], l[NW][kTile];
  __device__ WinFew() {}
  // This wave's tiles: number w, w + 4, .. of the list, each handed to f(j0) in LDS.
  template <typename F>
  __device__ __attribute__((always_inline)) inline void each(const WinTiles& tl, const float* K, const float* V, size_t ks,
                                                             size_t vs, int len, int w, int lane, F f) {
    if (w >= tl.n) return;
    typename C::Regs next;
    win_fetch<D, 1>(next, K, V, ks, vs, tl.first(w, kTile), len, lane);
    for (int n = w; n < tl.n; n += NW) {
      const int j0 = tl.first(n, kTile);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tiles have been read
      win_put<D, 1>(next, tiles.k[w], tiles.v[w], j0, len, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // and are there
      if (n + NW < tl.n) win_fetch<D, 1>(next, K, V, ks, vs, tl.first(n + NW, kTile), len, lane);
      f(j0);
    }
  }
  // The waves' sums, times f each, joined: wave w stores NCT of the row's 4 NCT pieces.  The tiles are free.
  __device__ __attribute__((always_inline)) inline void join(const typename C::Acc& acc, float f, int w, int lane) {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        parts[w][ct * 4 + e][lane] =
            f32x4{acc[ct][4 * e] * f, acc[ct][4 * e + 1] * f, acc[ct][4 * e + 2] * f, acc[ct][4 * e + 3] * f};
    __syncthreads();
  }
  __device__ __attribute__((always_inline)) inline void store(void* out, size_t row, float f, int w, int lane) const {
#pragma unroll
    for (int u = 0; u < NCT; ++u) {
      const int x = w * NCT + u;
      float o[4] = {};
#pragma unroll
      for (int y = 0; y < NW; ++y) {
        const f32x4 z = parts[y][x][lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += z[k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] *= f;
      store_out4<float>(out, row * D + x / 4 * kTile + row_of(x % 4 * 4, lane >> 5), o, true);
    }
  }
};

template <int D, typename A>
__global__ __launch_bounds__(kWave* kWinWaves) void hyb_win_fwd_few_kernel(A a, int wgs) {
  typedef WinF32<D, 1> C;
  __shared__ alignas(16) WinFew<D> sh;
  const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5;
  int g, x;
  const WinSeq<A> sq = win_of_queries<1>(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x);
  if (!me.any) return;  // uniform
  const int i = min(me.i0 + li, len - 1), end = min(me.i0 + kTile, len);
  const WinTiles tl(a, len, me.i0, end, kTile);
  const WinRow row(a, len, i), r0(a, len, me.i0), r1(a, len, end - 1);
  typename C::Ops qop;
  win_row_ops<D>(qop, (const float*)a.q + sq.q(me.h, D) + i * sq.qs(D), true, hh);
  const float scale = kLog2e / sqrtf((float)D);
  float m = kNoRef, l = 0.0f;
  typename C::Acc acc;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) acc[ct] = f32x16{};
  sh.each(tl, (const float*)a.k + sq.k(g, D), (const float*)a.v + sq.v(g, D), sq.ks(D), sq.vs(D), len, w, lane,
          [&](int j0) __attribute__((always_inline)) {
            win_take<D>(acc, m, l, sh.tiles.k[w], sh.tiles.v[w], qop, row, win_full(r0, r1, a.n_sinks, j0, kTile),
                        a.n_sinks, j0, scale, li, hh);
          });
  mma_settle<float>();
  if (hh == 0) sh.m[w][li] = m;
  __syncthreads();  // (and the tiles are free)
  float mm = sh.m[0][li];
#pragma unroll
  for (int y = 1; y < kWinWaves; ++y) mm = fmaxf(mm, sh.m[y][li]);
  const float f = __builtin_amdgcn_exp2f(m - mm);
  if (hh == 0) sh.l[w][li] = l * f;
  sh.join(acc, f, w, lane);
  l = 0.0f;
#pragma unroll
  for (int y = 0; y < kWinWaves; ++y) l += sh.l[y][li];
  if (me.i0 + li >= len) return;
  sh.store(a.out, sq.row(i) * a.s.Hq + me.h, 1.0f / l, w, lane);
  if (a.lse && w == 0 && hh == 0) a.lse[sq.lse(me.h, i)] = (mm + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, typename A>
__global__ __launch_bounds__(kWave* kWinWaves) void hyb_win_dq_few_kernel(A a, int wgs) {
  typedef WinF32<D, 1> C;
  __shared__ alignas(16) WinFew<D> sh;
  const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5, Hq = a.s.Hq;
  int g, x;
  const WinSeq<A> sq = win_of_queries<1>(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x);
  typename C::Acc acc;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) acc[ct] = f32x16{};
  if (me.any) {  // uniform
    const int i = min(me.i0 + li, len - 1), end = min(me.i0 + kTile, len);
    const WinTiles tl(a, len, me.i0, end, kTile);
    const WinRow row(a, len, i), r0(a, len, me.i0), r1(a, len, end - 1);
    typename C::Ops qop, dop;
    const size_t at = sq.dout(me.h, D) + (size_t)i * Hq * D;
    win_row_ops<D>(qop, (const float*)a.q + sq.q(me.h, D) + i * sq.qs(D), true, hh);
    win_row_ops<D>(dop, (const float*)a.dout + at, true, hh);
    float delta = 0.0f;
#pragma unroll
    for (int ks = 0; ks < C::KD; ++ks) delta += dop[ks] * ((const float*)a.out)[at + win_entry(ks, hh)];
    delta += xor32(delta);
    const float scale = kLog2e / sqrtf((float)D);
    const size_t st = sq.lse(me.h, i);
    const float lse = a.lse[st] * kLog2e;
    if (w == 0 && hh == 0 && me.i0 + li < len) a.ws[st] = delta;
    sh.each(tl, (const float*)a.k + sq.k(g, D), (const float*)a.v + sq.v(g, D), sq.ks(D), sq.vs(D), len, w, lane,
            [&](int j0) __attribute__((always_inline)) {
              win_take_dq<D>(acc, sh.tiles.k[w], sh.tiles.v[w], qop, dop, row, win_full(r0, r1, a.n_sinks, j0, kTile),
                             a.n_sinks, j0, scale, lse, delta, li, hh);
            });
    mma_settle<float>();
  }
  __syncthreads();  // (the tiles are free)
  sh.join(acc, 1.0f, w, lane);
  if (me.i0 + li >= sq.cap) return;  // rows past the length: zero
  sh.store(a.dq, sq.row(me.i0 + li) * Hq + me.h, me.i0 + li < len ? 1.0f / sqrtf((float)D) : 0.0f, w, lane);
}

// The queries that see some of the keys j0 .. j1 - 1 (j1 <= len): from q0 to q1 - 1.
struct WinQueries {
  int q0, q1;
  __device__ inline WinQueries(const WindowArgs& a, int len, int j0, int j1) {
    const int L = a.s.L;
    q0 = j0 / L * L;
    const long last = ((long)(j1 - 1) + a.window) / L * L + L;  // blocks that start by j1 - 1 + window
    q1 = j0 < a.n_sinks ? len : (int)min(last, (long)len);
  }
};

// dK, dV: a wave owns 32 keys, and loops over the queries of all heads of
// its KV head.
template <int D, typename A>
__global__ __launch_bounds__(kWave* kWinWaves) void hyb_win_dkv_kernel(A a, WinParts cut) {
  typedef WinF32<D> C;
  __shared__ alignas(16) typename C::Tile qt[2], dt[2];
  __shared__ alignas(16) float stats[2][2][kTile];  // lse (log2) and delta
  const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g;
  WinItem it;
  const WinSeq<A> sq = win_of_keys(a, cut, lane, g, it);
  const int len = sq.len;
  const int w0 = it.x * kWinKeys, j0 = w0 + w * kTile, j = j0 + li;  // first key of the workgroup, of the wave
  const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
  typename C::Acc dk, dv;
#pragma unroll
  for (int ct = 0; ct < C::NCT; ++ct) dk[ct] = dv[ct] = f32x16{};
  if (w0 < len) {  // uniform
    const WinQueries all(a, len, w0, min(w0 + kWinKeys, len));
    const int t0 = all.q0 / kTile, nq = (all.q1 + kTile - 1) / kTile - t0;
    const int first = (int)((long)nq * G * it.part / it.parts);
    const int nsteps = (int)((long)nq * G * (it.part + 1) / it.parts) - first;
    const WinKey mine(a, len, min(j, len - 1));
    typename C::Regs next;
    float nst = 0.0f;
    // Step n: the list's query tile first + n, of the group's heads in turn.
    auto tile = [&](int n) __attribute__((always_inline)) { return (t0 + (first + n) % nq) * kTile; };
    auto fetch = [&](int n) __attribute__((always_inline)) {
      const int h = g * G + (first + n) / nq, i0 = tile(n);
      win_fetch<D>(next, (const float*)a.q + sq.q(h, D), (const float*)a.dout + sq.dout(h, D), qs, (size_t)Hq * D, i0, len,
                   threadIdx.x);
      if (threadIdx.x < 2 * kTile) {
        const size_t at = sq.lse(h, min(i0 + (int)threadIdx.x % kTile, len - 1));
        nst = threadIdx.x < kTile ? a.lse[at] * kLog2e : a.ws[at];
      }
    };
    auto put = [&](int n) __attribute__((always_inline)) {
      const int buf = n & 1;
      win_put<D>(next, qt[buf], dt[buf], tile(n), len, threadIdx.x);
      if (threadIdx.x < 2 * kTile) (&stats[buf][0][0])[threadIdx.x] = nst;
    };
    if (nsteps > 0) fetch(0);
    typename C::Ops kop, vop;
    const size_t j1 = min(j, len - 1);
    win_row_ops<D>(kop, (const float*)a.k + sq.k(g, D) + j1 * ks_, j < len, hh);
    win_row_ops<D>(vop, (const float*)a.v + sq.v(g, D) + j1 * vs_, j < len, hh);
    const float scale = kLog2e / sqrtf((float)D);
    if (nsteps > 0) put(0);
    __syncthreads();
    for (int n = 0; n < nsteps; ++n) {
      const int i0 = tile(n), buf = n & 1;
      if (n + 1 < nsteps) fetch(n + 1);
      const WinRow r0(a, len, i0), r1(a, len, min(i0 + kTile, len) - 1);
      if (j0 < len && !win_none(r0, r1, a.n_sinks, j0, kTile)) {
        const f32x16 sc = win_rows_mma<D>(qt[buf], kop, li, hh);
        const f32x16 dp = win_rows_mma<D>(dt[buf], vop, li, hh);
        float p[16], ds[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = row_of(e, hh), i = i0 + r;
          const float x = __builtin_fmaf(sc[e], scale, -stats[buf][0][r]);
          p[e] = __builtin_amdgcn_exp2f(i >= mine.q0 && i < mine.q1 ? x : -INFINITY);
          ds[e] = p[e] * (dp[e] - stats[buf][1][r]);
        }
        win_cols_mma<D>(dv, dt[buf], p, li, hh);
        win_cols_mma<D>(dk, qt[buf], ds, li, hh);
        mma_settle<float>();
      }
      if (n + 1 < nsteps) put(n + 1);
      __syncthreads();
    }
  }
  if (j >= sq.cap) return;
  const size_t row = sq.row(j) * Hkv + g;
  const float fk = j < len ? 1.0f / sqrtf((float)D) : 0.0f, fv = j < len ? 1.0f : 0.0f;
  if (it.parts == 1) {
    win_store<float, D>(a.dk, row, dk, fk, hh, true);
    win_store<float, D>(a.dv, row, dv, fv, hh, true);
  } else {
    win_store<float, D>(it.sums<D>(a, cut), it.row(sq, 0, j, g), dk, fk, hh, true);
    win_store<float, D>(it.sums<D>(a, cut), it.row(sq, 1, j, g), dv, fv, hh, true);
  }
}

// ---- bf16 forward -----------------------------------------------------------
//
// The K and V tiles (32 rows) reach LDS by direct global->LDS copies into rings
// of R = 4 slots, chunk c of row t at c ^ swz(t) (V: vswz), so that the rows
// which one operand read touches fall in distinct banks.  A wave owns a unit of
// 32 queries; two workgroups share a CU, so that one's products run beside the
// other's weights.  (Two units per wave, which halves the LDS reads, leave one
// wave per SIMD and were slower: 8 x 8192 tokens, window 4096, 1935 us, where one took 1625.)
// Step n forms the scores of tile n + 1 while it takes the weights of tile n,
// then P V of tile n while it takes the maximum of tile n + 1: two independent
// chains, whose MFMAs and VALU instructions interleave.
template <int D>
struct WinRing {
  static constexpr int EPC = 8, CPR = D / EPC;
  static constexpr int RPI = kWave / CPR;  // rows per copy instruction
  static constexpr int RP256 = 256 / (D * 2);
  static constexpr int IK = kTile / RPI;   // copies per tile
  static constexpr int R = 4;
  __device__ static constexpr int swz(int t) { return (t / RP256) % CPR; }
  __device__ static constexpr int vswz(int t) { return 4 * ((t / RP256) % (CPR / 4)); }
};

// The reference of a query's weights moves only when a tile's maximum passes it
// by 2^8: until then weights are up to 2^8, which neither type minds, and the
// accumulators need no rescale.
constexpr float kRefSlack = 8.0f;

// Where workgroups are few and lists long, H = 2 halves of four waves take a unit's
// tiles in turn, each through rings of its own, and join their sums in LDS.  The halves
// have the same number of steps: one that is past the list's end copies the last tile
// again and hides it.
template <int D>
struct WinJoin {  // each half hands over the other's half of the entries
  static constexpr int NH = D / kTile / 2;
  float m[2][kWinWaves][kTile], l[2][kWinWaves][kTile];
  f32x4 x[2][kWinWaves][NH * 4][kWave];

  // Columns 32 NH O .. of a row's sums, for half O.
  template <int O>
  __device__ __attribute__((always_inline)) inline void give(int w, int lane, const f32x16 (&acc)[2 * NH]) {
#pragma unroll
    for (int ct = 0; ct < NH; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[O][w][ct * 4 + e][lane] = f32x4{acc[O * NH + ct][4 * e], acc[O * NH + ct][4 * e + 1],
                                          acc[O * NH + ct][4 * e + 2], acc[O * NH + ct][4 * e + 3]};
  }
  // Half O's own columns times f, plus the other's times fo.
  template <int O>
  __device__ __attribute__((always_inline)) inline void take(int w, int lane, f32x16 (&acc)[2 * NH], float f, float fo) const {
#pragma unroll
    for (int ct = 0; ct < NH; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 y = x[O][w][ct * 4 + e][lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[O * NH + ct][4 * e + k] = acc[O * NH + ct][4 * e + k] * f + y[k] * fo;
      }
  }
};
template <int D, int H, int R>
struct WinSmem {
  struct Rings {
    bf16 k[H][R][kTile * D], v[H][R][kTile * D];
  };
  struct None {};
  union {
    Rings rings;
    std::conditional_t<H == 2, WinJoin<D>, None> join;
  };
  __device__ WinSmem() {}
};
// A half's columns of a row.
template <int D, int H>
__device__ inline void win_store_half(void* out, size_t row, const f32x16 (&acc)[D / kTile], float f, int hh, bool f32,
                                      int half) {
  if constexpr (H == 1) {
    win_store<bf16, D>(out, row, acc, f, hh, f32);
  } else if (half == 0) {
    win_store<bf16, D, 0, D / kTile / 2>(out, row, acc, f, hh, f32);
  } else {
    win_store<bf16, D, D / kTile / 2, D / kTile>(out, row, acc, f, hh, f32);
  }
}

template <int D, int H, typename A>
__global__ __launch_bounds__(kWave* kWinWaves* H, 2) void hyb_win_ring_kernel(A a, int wgs) {
  typedef Mma<bf16> M;
  typedef M::op_t op_t;
  typedef WinRing<D> RG;
  constexpr int E = M::E, KW = M::KW, KD = D / KW, KL = kTile / KW, NCT = D / kTile, R = RG::R;
  constexpr int IPW = 2 * RG::IK / kWinWaves;  // copies per wave and step: waves 0, 1 K's, waves 2, 3 V's
  __shared__ alignas(16) WinSmem<D, H, R> sh;

  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = wave / kWinWaves, w = wave % kWinWaves;
  auto& kr = sh.rings.k[half];
  auto& vr = sh.rings.v[half];
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g, x;
  const WinSeq<A> sq = win_of_queries(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x * kWinWaves + w);
  const int first = x * kWinWaves / G * kTile, last = min(((x + 1) * kWinWaves - 1) / G * kTile + kTile, len);
  if (first >= len) return;  // uniform
  const WinTiles tl(a, len, first, last, kTile);
  const int ntiles = (tl.n + H - 1) / H;  // of each half: the list's every H-th
  auto key = [&](int n) __attribute__((always_inline)) { return tl.first(min(H * n + half, tl.n - 1), kTile); };
  const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
  const bf16* K = (const bf16*)a.k + sq.k(g, D);
  const bf16* V = (const bf16*)a.v + sq.v(g, D);

  op_t qop[KD];
  {
    const bf16* row = (const bf16*)a.q + sq.q(me.h, D) + min(me.i0 + li, len - 1) * qs + hh * E;
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) qop[ks] = load_op<bf16>(row + ks * KW);
  }
  float m = kNoRef, l = 0.0f;
  f32x16 acc[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  const WinRow row(a, len, min(me.i0 + li, len - 1));
  const WinRow r0(a, len, min(me.i0, len - 1)), r1(a, len, min(me.i0 + kTile, len) - 1);

  // Copies: lane's row and chunk of its wave's copies u; rows past the length
  // read the last row (masked below).
  int trow[IPW], tcol[IPW];
#pragma unroll
  for (int u = 0; u < IPW; ++u) {
    const int i = (w * IPW + u) % RG::IK;
    trow[u] = i * RG::RPI + lane / RG::CPR;
    const int pos = lane % RG::CPR;
    tcol[u] = (pos ^ (w < kWinWaves / 2 ? RG::swz(trow[u]) : RG::vswz(trow[u]))) * RG::EPC;
  }
  auto issue = [&](int n, bf16* dst) __attribute__((always_inline)) {
    if (n >= ntiles) return;
    const int j0 = key(n), left = len - 1 - j0;
    const size_t rs_ = w < kWinWaves / 2 ? ks_ : vs_;
    const bf16* base = (w < kWinWaves / 2 ? K : V) + (size_t)j0 * rs_;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(base), 0, (int)(kTile * rs_ * sizeof(bf16)), kBufferWord3);
#pragma unroll
    for (int u = 0; u < IPW; ++u)
      buf_to_lds16(rs, dst + (w * IPW + u) % RG::IK * RG::RPI * D,
                   (int)((min(trow[u], left) * (int)rs_ + tcol[u]) * sizeof(bf16)), 0);
  };
  // K of tile nk or V of tile nv, whichever this wave copies.
  auto issue_step = [&](int nk, bf16* dk, int nv, bf16* dv) __attribute__((always_inline)) {
    if (w < kWinWaves / 2)
      issue(nk, dk);
    else if (nv >= 0)
      issue(nv, dv);
  };

  const float scale = kLog2e / sqrtf((float)D);
  f32x16 sc;
  // Takes the scores of tile n: masks, maximum, reference.
  auto take = [&](int n, const f32x16& s) __attribute__((always_inline)) {
    sc = s;
    const int j0 = key(n);
    const bool over = H > 1 && H * n + half >= tl.n;
    if (over || !win_full(r0, r1, a.n_sinks, j0, kTile)) {  // uniform
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = (!over & row.sees(j0 + row_of(e, hh), a.n_sinks)) ? sc[e] : -INFINITY;
    }
    float mt = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
    mt = fmaxf(mt, xor32(mt)) * scale;
    if (__any(mt > m + kRefSlack)) {
      mma_settle<bf16>();
      const float mn = mt > m + kRefSlack ? mt : m;
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[ct][e] *= corr;
      m = mn;
    }
  };
  auto scores = [&](const bf16* kt) __attribute__((always_inline)) {
    op_t kop[KD];
#pragma unroll
    for (int ks = 0; ks < KD; ++ks)
      kop[ks] = load_op<bf16>(&kt[li * D + ((2 * ks + hh) ^ RG::swz(li)) * RG::EPC]);
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) s = M::mma(kop[ks], qop[ks], s);
    return s;
  };
  // Weights and P V of tile n (V in vt), scores of tile n + 1 (K in kt).
  auto compute = [&](auto lastc, int n, const bf16* kt, const bf16* vt) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(lastc)::value;
    f32x16 sn;
    if constexpr (!LAST) sn = scores(kt);
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -m));
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      s0 += p[e];
      s1 += p[e + 1];
    }
    l += s0 + s1;
    // The weights enter P V rounded to bf16 (each off by at most 2^-8 of itself, half
    // a step as any bf16 value; products of fp32 run at 1/16 of the rate); their sum
    // is over the unrounded ones, so lse carries none of it.
    op_t pop[KL];
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) pop[ks] = cvt_op<bf16>(&p[ks * E]);
    const int qi = lane & 15;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      const int col = ct * kTile + 16 * ((lane >> 4) & 1) + 4 * (qi & 3);
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) {
        const int r = 16 * ks + 4 * hh + qi / 4;
        const bf16* src = &vt[r * D + ((col / RG::EPC) ^ RG::vswz(qi / 4)) * RG::EPC + col % RG::EPC];
        acc[ct] = M::mma(lds_tr_op(src, src + 8 * D), pop[ks], acc[ct]);
      }
    }
    if constexpr (!LAST) take(n + 1, sn);
  };
  auto wait_step = [&](int later) __attribute__((always_inline)) {
    if (later >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * IPW) : "memory");
    else if (later == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * IPW) : "memory");
    else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPW) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  };
  const int ahead = w < kWinWaves / 2 ? 1 : 0;  // K runs a tile ahead
  auto step = [&](int n, auto S) __attribute__((always_inline)) {
    constexpr int SV = decltype(S)::value;
    wait_step(min(2, ntiles - 1 - n - ahead));
    lds_barrier_nodrain();  // K n+1 and V n visible; K n's and V n-1's slots free
    issue_step(n + R, kr[SV], n + R - 1, vr[(SV + R - 1) % R]);
    compute(std::false_type{}, n, kr[(SV + 1) % R], vr[SV]);
  };
  issue_step(0, kr[0], -1, nullptr);
  issue_step(1, kr[1], 0, vr[0]);
  issue_step(2, kr[2], 1, vr[1]);
  issue_step(3, kr[3], 2, vr[2]);
  wait_step(ahead ? min(3, ntiles - 1) : 3);
  lds_barrier_nodrain();
  take(0, scores(kr[0]));
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
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_barrier_nodrain();
  compute(std::true_type{}, ntiles - 1, nullptr, vr[ntiles - 1 - n]);

  l += xor32(l);
  if constexpr (H == 2) {
    mma_settle<bf16>();
    lds_barrier_nodrain();  // the rings are read
    if (hh == 0) {
      sh.join.m[half][w][li] = m;
      sh.join.l[half][w][li] = l;
    }
    if (half == 0)
      sh.join.template give<1>(w, lane, acc);
    else
      sh.join.template give<0>(w, lane, acc);
    lds_barrier_nodrain();
    const float mo = sh.join.m[1 - half][w][li], mm = fmaxf(m, mo);
    const float f = __builtin_amdgcn_exp2f(m - mm), fo = __builtin_amdgcn_exp2f(mo - mm);
    if (half == 0)
      sh.join.template take<0>(w, lane, acc, f, fo);
    else
      sh.join.template take<1>(w, lane, acc, f, fo);
    l = l * f + sh.join.l[1 - half][w][li] * fo;
    m = mm;
  }
  const int i = me.i0 + li;
  if (i >= len) return;
  win_store_half<D, H>(a.out, sq.row(i) * Hq + me.h, acc, 1.0f / l, hh, a.s.out_f32, half);
  if (a.lse && hh == 0 && half == 0) a.lse[sq.lse(me.h, i)] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// ---- bf16 gradient ----------------------------------------------------------
//
// Two kernels: dQ with delta and the rows' statistics (a wave owns 32 queries and
// loops over key tiles), then dK with dV (a wave owns 32 keys and loops over the
// query tiles of its KV head's heads).  Tiles come through rings as in the forward;
// here a tile is read both by rows and by columns (RowColTile).  8 x 2048 tokens: of a call's time
// dQ takes two fifths, dK and dV three (under a trace, which runs each call slower, 0.22 and 0.30 ms
// at best), their matrix cores busy 0.53 and 0.56 of the time.

// Statistics of a row for the dK, dV kernel, as operands of one more step of its
// products: lse sqrt(d) and delta, each as three bf16 pieces (24 bits), which
// that kernel multiplies by -1.  [B][Hq][Tp][16], Tp = T rounded up to a tile.
__host__ __device__ constexpr int win_tp(int T) { return (T + kTile - 1) / kTile * kTile; }
__device__ inline bf16x8 win_pieces(float x) {
  bf16x8 o = {};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    o[i] = (bf16)x;
    x -= (float)o[i];
  }
  return o;
}
template <int D, int H, typename A>
__global__ __launch_bounds__(kWave* kWinWaves* H, 2) void hyb_win_dq_ring_kernel(A a, int wgs) {
  typedef Mma<bf16> M;
  typedef M::op_t op_t;
  typedef RowColTile<D> WT;
  constexpr int E = M::E, KW = M::KW, KD = D / KW, KL = kTile / KW, NCT = D / kTile, R = 4;
  constexpr int IPW = 2 * WT::IK / kWinWaves;  // copies per wave and step: waves 0, 1 K's, waves 2, 3 V's
  __shared__ alignas(16) WinSmem<D, H, R> sh;

  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = wave / kWinWaves, w = wave % kWinWaves;
  auto& kr = sh.rings.k[half];
  auto& vr = sh.rings.v[half];
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g, x;
  const WinSeq<A> sq = win_of_queries(a, wgs, lane, g, x);
  const int len = sq.len;
  const WinUnit me = win_unit(a, len, g, x * kWinWaves + w);
  const int first = x * kWinWaves / G * kTile, last = min(((x + 1) * kWinWaves - 1) / G * kTile + kTile, len);
  f32x16 acc[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) acc[ct] = f32x16{};
  const int row = me.i0 + li;
  // The statistics of row i, a half in each of its lanes; zero past the length.
  const auto put_stats = [&](float e, float s) __attribute__((always_inline)) {
    if (me.i0 < sq.cap && half == 0)
      reinterpret_cast<bf16x8*>(a.ws)[sq.stats(me.h, row) * 2 + hh] =
          win_pieces(row < len ? (hh == 0 ? e : s) : 0.0f);
  };
  if (first >= len) put_stats(0.0f, 0.0f);
  if (first < len) {  // uniform
    const WinTiles tl(a, len, first, last, kTile);
    const int ntiles = (tl.n + H - 1) / H;
    auto key = [&](int n) __attribute__((always_inline)) { return tl.first(min(H * n + half, tl.n - 1), kTile); };
    const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
    const bf16* K = (const bf16*)a.k + sq.k(g, D);
    const bf16* V = (const bf16*)a.v + sq.v(g, D);
    const int i = min(row, len - 1);
    const WinRow mine(a, len, i), r0(a, len, min(me.i0, len - 1)), r1(a, len, min(me.i0 + kTile, len) - 1);
    const WT wt(lane);
    op_t qop[KD], dop[KD];
    float delta = 0.0f;
    {
      const size_t at = sq.dout(me.h, D) + (size_t)i * Hq * D + hh * E;
      const bf16* qrow = (const bf16*)a.q + sq.q(me.h, D) + i * qs + hh * E;
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) {
        qop[ks] = load_op<bf16>(qrow + ks * KW);
        dop[ks] = load_op<bf16>((const bf16*)a.dout + at + ks * KW);
      }
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) {
        const op_t o = load_op<bf16>((const bf16*)a.out + at + ks * KW);
#pragma unroll
        for (int e = 0; e < E; ++e) delta += (float)o[e] * (float)dop[ks][e];
      }
      delta += xor32(delta);
    }
    const float scale = kLog2e / sqrtf((float)D);
    const float nat = a.lse[sq.lse(me.h, i)], lse = nat * kLog2e;
    put_stats(nat * sqrtf((float)D), delta);

    int trow[IPW], tcol[IPW];
#pragma unroll
    for (int u = 0; u < IPW; ++u) {
      trow[u] = (w * IPW + u) % WT::IK * WT::RPI + lane / WT::CPR;
      tcol[u] = (lane % WT::CPR ^ WT::swz(trow[u])) * WT::EPC;
    }
    auto issue = [&](int n, bf16* dk, bf16* dv) __attribute__((always_inline)) {
      if (n >= ntiles) return;
      const bool isk = w < kWinWaves / 2;
      bf16* dst = isk ? dk : dv;
      const int j0 = key(n), left = len - 1 - j0;
      const size_t rs_ = isk ? ks_ : vs_;
      const bf16* base = (isk ? K : V) + (size_t)j0 * rs_;
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(base), 0, (int)(kTile * rs_ * sizeof(bf16)), kBufferWord3);
#pragma unroll
      for (int u = 0; u < IPW; ++u)
        buf_to_lds16(rs, dst + (w * IPW + u) % WT::IK * WT::RPI * D,
                     (int)((min(trow[u], left) * (int)rs_ + tcol[u]) * sizeof(bf16)), 0);
    };
    f32x16 sc, dp;
    // Scores and dP of tile n, masked.
    auto products = [&](const bf16* kt, const bf16* vt, f32x16& s, f32x16& d) __attribute__((always_inline)) {
      s = f32x16{};
      d = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) s = M::mma(wt.row_op(kt, ks), qop[ks], s);
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) d = M::mma(wt.row_op(vt, ks), dop[ks], d);
    };
    auto take = [&](int n, const f32x16& s, const f32x16& d) __attribute__((always_inline)) {
      sc = s;
      dp = d;
      const int j0 = key(n);
      const bool over = H > 1 && H * n + half >= tl.n;
      if (over || !win_full(r0, r1, a.n_sinks, j0, kTile)) {  // uniform
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = (!over & mine.sees(j0 + row_of(e, hh), a.n_sinks)) ? sc[e] : -INFINITY;
      }
    };
    auto compute = [&](auto lastc, int n, const bf16* kn, const bf16* vn, const bf16* kt) __attribute__((always_inline)) {
      constexpr bool LAST = decltype(lastc)::value;
      f32x16 sn, dn;
      if constexpr (!LAST) products(kn, vn, sn, dn);
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e)
        ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -lse)) * (dp[e] - delta);
      op_t sop[KL];  // (dS rounded to bf16 for its product, as the weights of the forward)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) sop[ks] = cvt_op<bf16>(&ds[ks * E]);
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int ks = 0; ks < KL; ++ks) acc[ct] = M::mma(wt.col_op(kt, ct, ks), sop[ks], acc[ct]);
      if constexpr (!LAST) take(n + 1, sn, dn);
    };
    // Tile n + 1 is read at step n, by rows, and tile n by columns; tile n + 3
    // goes to the slot of tile n - 1.
    auto step = [&](int n, auto S) __attribute__((always_inline)) {
      constexpr int SV = decltype(S)::value;
      if (n + 2 < ntiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPW) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier_nodrain();
      issue(n + 3, kr[(SV + 3) % R], vr[(SV + 3) % R]);
      compute(std::false_type{}, n, kr[(SV + 1) % R], vr[(SV + 1) % R], kr[SV]);
    };
    issue(0, kr[0], vr[0]);
    issue(1, kr[1], vr[1]);
    issue(2, kr[2], vr[2]);
    if (ntiles > 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * IPW) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier_nodrain();
    {
      f32x16 s, d;
      products(kr[0], vr[0], s, d);
      take(0, s, d);
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
    compute(std::true_type{}, ntiles - 1, nullptr, nullptr, kr[ntiles - 1 - n]);
    if constexpr (H == 2) {
      mma_settle<bf16>();
      lds_barrier_nodrain();  // the rings are read
      if (half == 0)
        sh.join.template give<1>(w, lane, acc);
      else
        sh.join.template give<0>(w, lane, acc);
      lds_barrier_nodrain();
      if (half == 0)
        sh.join.template take<0>(w, lane, acc, 1.0f, 1.0f);
      else
        sh.join.template take<1>(w, lane, acc, 1.0f, 1.0f);
    }
  }
  if (row >= sq.cap) return;  // rows past the length: zero
  win_store_half<D, H>(a.dq, sq.row(row) * Hq + me.h, acc, row < len ? 1.0f / sqrtf((float)D) : 0.0f, hh,
                       a.s.out_f32, half);
}

// A workgroup owns 128 keys, a wave 32 of them.  With H = 2 it has two halves of
// four waves, which take the query tiles in turn and join their sums in LDS at the
// end: at d = 128, so that two waves share a SIMD with the LDS of one workgroup (dK and
// dV take 128 registers, K 32, the scores and dP 32; V is read from LDS); at d = 64, where
// three workgroups of four waves fit a CU, where there are fewer (win_cut).
template <int D, int H, typename A>
__global__ __launch_bounds__(kWave * 4 * H, 2) void hyb_win_dkv_ring_kernel(A a, WinParts cut) {
  typedef Mma<bf16> M;
  typedef M::op_t op_t;
  typedef RowColTile<D> WT;
  constexpr int E = M::E, KW = M::KW, KD = D / KW, KL = kTile / KW, NCT = D / kTile, R = 3;
  constexpr int IPQ = 2 * WT::IK / 4;  // a half's copies per wave and step: two waves Q's, two dO's
  constexpr int IPW = IPQ + 1;         // and a quarter of the statistics each
  struct alignas(16) Slot {
    bf16 q[kTile * D], d[kTile * D], st[kTile * 16];
  };
  struct Loop {
    Slot ring[H][R];
    bf16 v[4][kTile * D];
  };
  struct Join {  // (the other half's dK or dV)
    f32x4 x[H == 2 ? 2 : 0][4][NCT * 4][kWave];
  };
  union Smem {
    Loop loop;
    Join join;
    __device__ Smem() {}
  };
  __shared__ Smem sh;

  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = wave >> 2, w = wave & 3;
  const int li = lane & 31, hh = lane >> 5;
  const int Hq = a.s.Hq, Hkv = a.s.Hkv, G = Hq / Hkv;
  int g;
  WinItem it;
  const WinSeq<A> sq = win_of_keys(a, cut, lane, g, it);
  const int len = sq.len;
  const int w0 = it.x * kWinKeys, j0 = w0 + w * kTile, j = j0 + li;
  f32x16 acc[2][NCT];  // dK, dV
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) acc[0][ct] = acc[1][ct] = f32x16{};
  if (w0 < len) {  // uniform
    const size_t qs = sq.qs(D), ks_ = sq.ks(D), vs_ = sq.vs(D);
    // query tiles t0 .. t0 + nq - 1 of every head, of which this part takes
    // ntiles from first on, a half every H-th
    const WinQueries all(a, len, w0, min(w0 + kWinKeys, len));
    const int t0 = all.q0 / kTile, nq = (all.q1 + kTile - 1) / kTile - t0;
    const int first = (int)((long)nq * G * it.part / it.parts);
    const int ntiles = (int)((long)nq * G * (it.part + 1) / it.parts) - first;
    const int nsteps = (ntiles + H - 1) / H, mysteps = (ntiles + H - 1 - half) / H;
    const WinKey mine(a, len, min(j, len - 1));
    // query tiles that every key of the wave is seen by: f0 <= i0 and i0 + 32 <= f1
    const int jl = max(min(j0 + kTile, len) - 1, 0);
    const int f0 = WinKey(a, len, jl).q0, f1 = WinKey(a, len, min(max(j0, a.n_sinks), jl)).q1;
    const WT wt(lane);
    // this half's share of V: 4 / H of the keys' tiles, a copy per wave and round
#pragma unroll
    for (int u = 0; u < WT::IK / H; ++u) {
      const int c = u * 4 + w, t = 4 / H * half + c / WT::IK, r = c % WT::IK * WT::RPI + lane / WT::CPR;
      const bf16* src = (const bf16*)a.v + sq.v(g, D) + min(w0 + t * kTile + r, len - 1) * vs_ +
                        (lane % WT::CPR ^ WT::swz(r)) * WT::EPC;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                       (__attribute__((address_space(3))) void*)(sh.loop.v[t] + c % WT::IK * WT::RPI * D),
                                       16, 0, 0);
    }
    op_t kop[KD];
    {
      const size_t at = sq.k(g, D) + min(j, len - 1) * ks_ + hh * E;
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) kop[ks] = load_op<bf16>((const bf16*)a.k + at + ks * KW);
    }
    op_t ms = {}, md = {};  // -1 for the three pieces of lse (hh = 0), of delta (hh = 1)
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      ms[e] = (bf16)(hh == 0 ? -1.0f : 0.0f);
      md[e] = (bf16)(hh == 1 ? -1.0f : 0.0f);
    }
    const float scale = kLog2e / sqrtf((float)D);

    int trow[IPQ], tcol[IPQ];
#pragma unroll
    for (int u = 0; u < IPQ; ++u) {
      trow[u] = (w * IPQ + u) % WT::IK * WT::RPI + lane / WT::CPR;
      tcol[u] = (lane % WT::CPR ^ WT::swz(trow[u])) * WT::EPC;
    }
    // Head and query tile of this half's next copies and next products.
    int inh = g * G + (first + half) / nq, inq = (first + half) % nq, cq = inq;
    auto issue = [&](int n, Slot& s) __attribute__((always_inline)) {
      if (n >= mysteps) return;
      const int i0 = (t0 + inq) * kTile, left = len - 1 - i0;
      const bool isq = w < 2;
      const size_t rs_ = isq ? qs : (size_t)Hq * D;
      const bf16* base = (const bf16*)(isq ? a.q : a.dout) + (isq ? sq.q(inh, D) : sq.dout(inh, D)) + (size_t)i0 * rs_;
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(base), 0, (int)(kTile * rs_ * sizeof(bf16)), kBufferWord3);
      bf16* dst = isq ? s.q : s.d;
#pragma unroll
      for (int u = 0; u < IPQ; ++u)
        buf_to_lds16(rs, dst + (w * IPQ + u) % WT::IK * WT::RPI * D,
                     (int)((min(trow[u], left) * (int)rs_ + tcol[u]) * sizeof(bf16)), 0);
      const float* st = (const float*)a.ws + sq.stats(inh, i0) * 8 + w * kWave + lane;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)st,
                                       (__attribute__((address_space(3))) void*)((float*)s.st + w * kWave), 4, 0, 0);
      inq += H;
      while (inq >= nq) inq -= nq, ++inh;
    };
    auto compute = [&](const Slot& s) __attribute__((always_inline)) {
      const op_t st = *reinterpret_cast<const op_t*>(&s.st[li * 16 + hh * 8]);
      f32x16 sc = M::mma(st, ms, f32x16{}), dp = M::mma(st, md, f32x16{});
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) sc = M::mma(wt.row_op(s.q, ks), kop[ks], sc);
#pragma unroll
      for (int ks = 0; ks < KD; ++ks) dp = M::mma(wt.row_op(s.d, ks), wt.row_op(sh.loop.v[w], ks), dp);
      const int i0 = (t0 + cq) * kTile;
      if (!(i0 >= f0 && i0 + kTile <= f1)) {  // uniform
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int i = i0 + row_of(e, hh);
          sc[e] = i >= mine.q0 && i < mine.q1 ? sc[e] : -INFINITY;
        }
      }
      cq += H;
      while (cq >= nq) cq -= nq;
      op_t pop[KL], sop[KL];  // (P and dS rounded to bf16 for their products, as in the forward)
#pragma unroll
      for (int ks = 0; ks < KL; ++ks) {
        float p[E], ds[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          p[e] = __builtin_amdgcn_exp2f(sc[ks * E + e] * scale);
          ds[e] = p[e] * dp[ks * E + e];
        }
        pop[ks] = cvt_op<bf16>(p);
        sop[ks] = cvt_op<bf16>(ds);
      }
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int ks = 0; ks < KL; ++ks) {
          acc[1][ct] = M::mma(wt.col_op(s.d, ct, ks), pop[ks], acc[1][ct]);
          acc[0][ct] = M::mma(wt.col_op(s.q, ct, ks), sop[ks], acc[0][ct]);
        }
    };
    // Tile n + 2 of the half goes to the slot of tile n - 1.
    auto step = [&](int n, auto S) __attribute__((always_inline)) {
      constexpr int SV = decltype(S)::value;
      if (n + 1 < mysteps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPW) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier_nodrain();
      issue(n + 2, sh.loop.ring[half][(SV + 2) % R]);
      if (n < mysteps) compute(sh.loop.ring[half][SV]);
    };
    issue(0, sh.loop.ring[half][0]);
    issue(1, sh.loop.ring[half][1]);
    for (int n = 0; n < nsteps; n += R) {
      step(n, std::integral_constant<int, 0>{});
      if (n + 1 < nsteps) step(n + 1, std::integral_constant<int, 1>{});
      if (n + 2 < nsteps) step(n + 2, std::integral_constant<int, 2>{});
    }
    // (a part without query tiles, where keys have fewer than parts, has taken no
    // step, and its copies of V may be on their way into what the sums take over)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (H == 2) {
      // The halves' sums: each hands over one of dK and dV and keeps the other.
      lds_barrier_nodrain();
#pragma unroll
      for (int o = 0; o < 2; ++o)
        if (o != half)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sh.join.x[o][w][ct * 4 + e][lane] = f32x4{acc[o][ct][4 * e], acc[o][ct][4 * e + 1], acc[o][ct][4 * e + 2],
                                                        acc[o][ct][4 * e + 3]};
      lds_barrier_nodrain();
#pragma unroll
      for (int o = 0; o < 2; ++o)
        if (o == half)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4 y = sh.join.x[o][w][ct * 4 + e][lane];
#pragma unroll
              for (int k = 0; k < 4; ++k) acc[o][ct][4 * e + k] += y[k];
            }
    }
  }
  if (j >= sq.cap) return;
  const size_t row = sq.row(j) * Hkv + g;
#pragma unroll
  for (int o = 0; o < 2; ++o)
    if (H == 1 || o == half) {
      const float f = j >= len ? 0.0f : o == 0 ? 1.0f / sqrtf((float)D) : 1.0f;
      if (it.parts == 1)
        win_store<bf16, D>(o == 0 ? a.dk : a.dv, row, acc[o], f, hh, a.s.out_f32);
      else
        win_store<bf16, D>(it.sums<D>(a, cut), it.row(sq, o, j, g), acc[o], f, hh, true);
    }
}

// dK and dV from the parts' sums, in order; four entries per thread.  Keys from
// `end` on have one part, written in place.
template <typename T, int D>
__global__ __launch_bounds__(256) void hyb_win_sum_kernel(WindowArgs a, WinParts cut, int end) {
  const size_t per = (size_t)a.s.Hkv * D / 4, n = (size_t)a.s.B * end * per;
  for (size_t x = (size_t)blockIdx.x * 256 + threadIdx.x; x < 2 * n; x += (size_t)gridDim.x * 256) {
    const int o = x >= n;
    const size_t y = x - o * n, bj = y / per, c = y % per;
    const int b = (int)(bj / end), j = (int)(bj % end);
    const bool sink = j < cut.ns * kWinKeys;
    const int parts = sink ? cut.ps : cut.p, span = sink ? cut.ns * kWinKeys : a.T;
    const f32x4* src = reinterpret_cast<const f32x4*>(a.sums) + (sink ? 0 : cut.sink_rows() * 2 * a.s.B * per) +
                       (((size_t)o * a.s.B + b) * span + j) * per + c;
    f32x4 s = {};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) s += src[(size_t)2 * a.s.B * span * per * p];
    const float v[4] = {s[0], s[1], s[2], s[3]};
    store_out4<T>(o ? a.dv : a.dk, 4 * (((size_t)b * a.T + j) * per + c), v, a.s.out_f32);
  }
}

// Workgroups of a (request, KV head): its queries' units, one per wave.
static int win_wgs(const WindowArgs& a) {
  const long units = ((long)a.T + kTile - 1) / kTile * (a.s.Hq / a.s.Hkv);
  return (int)((units + kWinWaves - 1) / kWinWaves);
}

// Whether n workgroups' units are taken in two halves (bf16): where at most two
// workgroups of one half would share a CU and the longest lists have 32 tiles and
// more (1 x 2048 tokens, 16 heads of d = 128, every earlier block: 256 workgroups, 51 us
// in one half, now 41; 2 x 2048, 512 workgroups, 58 and 51; 1 x 4096, 8 heads of d = 64, 67
// and 54; but a window of 512 for 1 x 4096, 8 heads, 17.5 and 18.2, and 1024 workgroups of
// 1 x 8192, window 4096, 245 both).
static bool win_halves(const WindowArgs& a, int n) {
  const long seen = std::min<long>(a.T, (long)a.window + std::min(a.n_sinks, a.T) + a.s.L);
  return n <= 512 && seen >= 32 * kTile;
}
// Packed (T is the mean length): the longest lists come first and end last.  (us of a forward in one
// half and in two: 3 sequences of 375 to 1126, 12 heads of d = 128, 33 and 29; 12 of 75 to 900, 8 heads,
// 33 and 27, at d = 64 22 and 20; 4 of 375 to 1500, 16 heads, 49 and 41; 1 of 400 15.3 and 15.6; but 20
// of 15 to 300 16.5 and 23.)
static bool win_halves(const PackedArgs& a, int n) {
  const long seen = std::min<long>(a.T, (long)a.window + std::min(a.n_sinks, a.T) + a.s.L);
  return n <= 512 && seen >= 10 * kTile;
}

// The grids of the queries' and keys' workgroups: `wgs` and `keys` per (request, KV head), or
// packed per KV head; `busy` of the queries' are at work.
template <typename A>
struct WinGrid;
template <>
struct WinGrid<WindowArgs> {
  int wgs, n, busy, heads;
  explicit WinGrid(const WindowArgs& a) : wgs(win_wgs(a)), n(a.s.B * a.s.Hkv * wgs), busy(n), heads(a.s.B * a.s.Hkv) {}
  int items(const WindowArgs&, const WinParts& cut) const { return cut.items(); }
};
template <>
struct WinGrid<PackedArgs> {
  int wgs, n, busy, heads;
  explicit WinGrid(const PackedArgs& a, int U = kWinWaves) : heads(a.s.Hkv) {
    wgs = (int)win_packed_queries(a.N, a.s.B + 1, a.s.Hq / a.s.Hkv, U);
    n = wgs * heads;
    busy = (int)std::min<long>(n, ((long)a.N / kTile + a.s.B / 2) * a.s.Hq / U);
  }
  int items(const PackedArgs& a, const WinParts& cut) const { return (int)win_packed_keys(a.N, a.s.B + 1) * cut.p; }
};

template <int D, typename A>
static hipError_t win_ring_go(const A& a, hipStream_t st) {
  const WinGrid<A> gr(a);
  const dim3 grid((unsigned)gr.n);
  if (win_halves(a, gr.busy))
    hipLaunchKernelGGL((hyb_win_ring_kernel<D, 2, A>), grid, dim3(kWave * kWinWaves * 2), 0, st, a, gr.wgs);
  else
    hipLaunchKernelGGL((hyb_win_ring_kernel<D, 1, A>), grid, dim3(kWave * kWinWaves), 0, st, a, gr.wgs);
  return hipGetLastError();
}

// Whether n units of packed sequences (fp32) have a workgroup each: where lists are long and units
// few; at d = 128 one such workgroup fits a CU, at 64 two.  (us of a forward and a gradient so and
// otherwise.  d = 64: 5 sequences of 140 to 701, 8 heads, 545 units, 32 and 58, 141 and 189; 1 of 2048,
// 516, 74 and 103, 219 and 363; 16 of 64 to 1024, 2240, 99 and 117, 351 and 377; but 16 of 128 to
// 2048, 4416, 295 and 273, and 20 of 5 to 100, 18.7 and 15.7.  d = 128: 2 of 175 and 350, 16 heads,
// 278, 28 and 41, 99 and 149; 3 of 192, 8 heads, 156, 21 and 24, 70 and 95; 4 of 128 to 512, 672, 52 and 78,
// 177 and 228; but 16 of 44 to 700, 1550, 144 and 106, 447 and 417.)
static bool win_few(const PackedArgs& a, int n) {
  const long seen = std::min<long>(a.T, (long)a.window + std::min(a.n_sinks, a.T) + a.s.L);
  return (n <= 640 && seen >= 4 * kTile) || (n <= (a.s.D == 64 ? 2560 : 1024) && seen >= 8 * kTile);
}

template <int D, typename A>
static hipError_t win_prefill_f32_go(const A& a, hipStream_t st) {
  const WinGrid<A> gr(a);
  const dim3 grid((unsigned)gr.n);
  if constexpr (std::is_same_v<A, PackedArgs>) {
    const WinGrid<A> one(a, 1);
    if (win_few(a, one.busy)) {
      hipLaunchKernelGGL((hyb_win_fwd_few_kernel<D, A>), dim3((unsigned)one.n), dim3(kWave * kWinWaves), 0, st, a, one.wgs);
      return hipGetLastError();
    }
    // Two units per workgroup while those have a CU each: a SIMD then has one wave of a
    // step's products, not two (32 heads of d = 128, 1 sequence of 125: 26 us with four
    // units, 18 with two).
    const WinGrid<A> two(a, 2);
    if (two.busy <= 256) {
      hipLaunchKernelGGL((hyb_win_fwd_kernel<D, 2, A, 2>), dim3((unsigned)two.n), dim3(kWave * 4), 0, st, a, two.wgs);
      return hipGetLastError();
    }
  }
  // Two halves at d = 128, where one workgroup fits a CU either way (8 x 4096 tokens,
  // 16 heads, window 500, 1404 us with one, now 1300; 1 x 1024, 159 and 144), and at
  // d = 64, where three of one half fit, while workgroups are few (1 x 3000 tokens, 192
  // of them, 260 and 215; 2 x 2048, 512, 231 and 165; of 4096 616, and 684 in halves).
  bool halves = true;
  if constexpr (D == 64) {
    halves = gr.busy <= 512;
    if (!halves) hipLaunchKernelGGL((hyb_win_fwd_kernel<D, 1, A>), grid, dim3(kWave * kWinWaves), 0, st, a, gr.wgs);
  }
  if (halves)
    hipLaunchKernelGGL((hyb_win_fwd_kernel<D, 2, A>), grid, dim3(kWave * kWinWaves * 2), 0, st, a, gr.wgs);
  return hipGetLastError();
}

// The cut: parts and, on bf16 at d = 64, halves, with the least estimated time (us): a
// list costs its start and end (`fixed`) besides its query tiles (`unit` each), the chip
// takes a workgroup per CU at a time (on bf16 at d = 64 without halves several share one),
// and more parts than one cost the sums' traffic and a launch.  The numbers are fitted to 23
// shapes of bf16 and 16 of fp32 with up to 16 parts, where what this takes is within 2%
// of the best on average and 11% in each.  (d = 128, 2 x 1024 tokens, window 200, 16 and 4 heads:
// 60 us in 1 part, 47 in 3, 46 in 4, which are 256 lists, 58 in 5; fp32 538, 246, 208, 259, where
// the estimate takes 8, 230.  d = 64, 2 x 3001, window 511, 8 and 2 heads: no halves, 1 to 5 parts
// 89, 65, 56, 58, 56; halves, 67, 54, 60, 61, 58.)
// The sinks' keys are cut into parts as long as the others', as long as those
// are at most 16 per (request, KV head) and 512 in all.
static int win_sink_parts(const Shape& s) { return (int)std::min<long>(16, 512 / std::max<long>(1, (long)s.B * s.Hkv)); }
static int win_most_parts(const Shape& s, int T) {
  const long all = (long)s.B * s.Hkv * ((T + kWinKeys - 1) / kWinKeys);
  const long every = ((long)T + kTile - 1) / kTile * (s.Hq / s.Hkv);
  return (int)std::max<long>(1, std::min<long>({16, 1024 / all, every / 8}));
}
static WinParts win_cut(const Shape& s, int T, int window, int n_sinks) {
  const int G = s.Hq / s.Hkv;
  WinParts c;
  c.wgs = (T + kWinKeys - 1) / kWinKeys;
  c.ns = std::min(c.wgs, (std::min(n_sinks, T) + kWinKeys - 1) / kWinKeys);
  const double all = (double)s.B * s.Hkv * c.wgs, every = std::ceil(T / 32.0);
  const double seen = std::min(every, std::ceil(((double)window + s.L + kWinKeys) / kTile) + 1);  // tiles of a head
  const double mean = seen - seen * seen / (2 * every);  // (the last keys' lists end early)
  const bool f32 = s.dtype != 1;
  const double launch = 4.5, sum = (double)s.B * T * s.Hkv * s.D * (f32 ? 3.5e-6 : 2.5e-6);
  double best = 0;
  c.p = 0;
  for (int h = f32 || s.D == 64 ? 1 : 2; h <= (f32 ? 1 : 2); ++h) {
    const double unit = f32 ? 6.0 * s.D / 64 : s.D == 128 ? 0.75 : h == 1 ? 0.65 : 0.4;
    const double fixed = f32 || s.D == 128 ? 6.0 : h == 1 ? 1.0 : 2.5;
    for (int p = 1; p <= win_most_parts(s, T); ++p) {
      const double rounds = f32 || h == 2 ? std::ceil(all * p / 256) : std::max(1.0, all * p / 450);
      const double t = rounds * fixed + G * unit / p * std::max(seen, rounds * mean) + (p > 1 ? launch + p * sum : 0);
      if (c.p == 0 || t < best) {
        best = t;
        c.p = p;
        c.halves = h == 2;
      }
    }
  }
  const int each = (int)std::ceil(seen * G / c.p);
  c.ps = c.p;
  if (c.ns > 0 && every * G >= 2 * each)
    c.ps = (int)std::max<long>(c.p, std::min<long>((long)((every * G + each - 1) / each), win_sink_parts(s) / c.ns));
  return c;
}
// bf16: the rows' statistics; fp32: delta.
static size_t win_stats_bytes(const Shape& s, int T) {
  return s.dtype == 1 ? (size_t)s.B * s.Hq * win_tp(T) * 32 : ((size_t)s.B * s.Hq * T * sizeof(float) + 255) / 256 * 256;
}
// Partial sums at most, for any window and number of sinks: the sinks'
// workgroups times their parts are within win_sink_parts, or have p parts as every
// workgroup (one workgroup's keys see one list, with or without sinks).
static size_t win_sums_bytes(const Shape& s, int T) {
  const int wgs = (T + kWinKeys - 1) / kWinKeys, p = win_most_parts(s, T), sp = win_sink_parts(s);
  const long sinks = wgs > 1 && sp > 1 ? sp : 0;
  const long tiles = p > 1 ? std::max((long)wgs * p, sinks) : sinks;
  return (size_t)(tiles * kWinKeys + (p > 1 ? (long)p * T : 0)) * 2 * s.B * s.Hkv * s.D * sizeof(float);
}

// The gradient's kernels but the last.
template <typename T, int D, typename A>
static void win_backward_kernels(const A& a, const WinParts& cut, hipStream_t st) {
  const WinGrid<A> gr(a);
  const dim3 gq((unsigned)gr.n), gk((unsigned)(gr.heads * gr.items(a, cut)));
  if constexpr (sizeof(T) == 2) {
    // (dQ in halves at d = 64 only, 1 x 4096 tokens as above 139 and 114 us with dK, dV;
    // at d = 128 two halves need more registers than there are, and were no faster)
    bool halves = false;
    if constexpr (D == 64) {
      halves = win_halves(a, gr.busy);
      if (halves) hipLaunchKernelGGL((hyb_win_dq_ring_kernel<D, 2, A>), gq, dim3(kWave * kWinWaves * 2), 0, st, a, gr.wgs);
    }
    if (!halves) hipLaunchKernelGGL((hyb_win_dq_ring_kernel<D, 1, A>), gq, dim3(kWave * kWinWaves), 0, st, a, gr.wgs);
    if constexpr (D == 64) {
      if (!cut.halves) hipLaunchKernelGGL((hyb_win_dkv_ring_kernel<D, 1, A>), gk, dim3(kWave * 4), 0, st, a, cut);
    }
    if (D == 128 || cut.halves) hipLaunchKernelGGL((hyb_win_dkv_ring_kernel<D, 2, A>), gk, dim3(kWave * 8), 0, st, a, cut);
  } else {
    bool few = false;
    if constexpr (std::is_same_v<A, PackedArgs>) {
      const WinGrid<A> one(a, 1);
      few = win_few(a, one.busy);
      if (few)
        hipLaunchKernelGGL((hyb_win_dq_few_kernel<D, A>), dim3((unsigned)one.n), dim3(kWave * kWinWaves), 0, st, a, one.wgs);
    }
    if (!few) hipLaunchKernelGGL((hyb_win_dq_kernel<D, A>), gq, dim3(kWave * kWinWaves), 0, st, a, gr.wgs);
    hipLaunchKernelGGL((hyb_win_dkv_kernel<D, A>), gk, dim3(kWave * kWinWaves), 0, st, a, cut);
  }
}
// The sums of the parts of keys 0 .. end - 1 of every sequence.
template <typename T, int D>
static hipError_t win_backward_sums(const WindowArgs& a, const WinParts& cut, int end, hipStream_t st) {
  if (end > 0) {
    const long n = (long)a.s.B * end * a.s.Hkv * D / 2;
    hipLaunchKernelGGL((hyb_win_sum_kernel<T, D>), dim3((unsigned)std::min<long>((n + 255) / 256, 4096)), dim3(256), 0,
                       st, a, cut, end);
  }
  return hipGetLastError();
}

template <typename T, int D>
static hipError_t win_backward_go(WindowArgs a, hipStream_t st) {
  const WinParts cut = win_cut(a.s, a.T, a.window, a.n_sinks);
  a.sums = (float*)((char*)a.ws + win_stats_bytes(a.s, a.T));
  // (what the workspace was sized for, whatever window and n_sinks are)
  if ((size_t)cut.rows(a.T) * 2 * a.s.B * a.s.Hkv * D * sizeof(float) > win_sums_bytes(a.s, a.T))
    return hipErrorInvalidValue;
  win_backward_kernels<T, D>(a, cut, st);
  return win_backward_sums<T, D>(a, cut, cut.p > 1 ? a.T : cut.ps > 1 ? std::min(cut.ns * kWinKeys, a.T) : 0, st);
}

hipError_t launch_window_prefill(const WindowArgs& a, hipStream_t st) {
  if (a.s.dtype == 1) return a.s.D == 64 ? win_ring_go<64>(a, st) : win_ring_go<128>(a, st);
  return a.s.D == 64 ? win_prefill_f32_go<64>(a, st) : win_prefill_f32_go<128>(a, st);
}

hipError_t launch_window_backward(const WindowArgs& a, hipStream_t st) {
  if (a.s.dtype == 1) return a.s.D == 64 ? win_backward_go<bf16, 64>(a, st) : win_backward_go<bf16, 128>(a, st);
  return a.s.D == 64 ? win_backward_go<float, 64>(a, st) : win_backward_go<float, 128>(a, st);
}

// ---- packed sequences ---------------------------------------------------------

// Mean length, for the choices that the host makes.
static int packed_mean(const Shape& s, int N) { return std::max(1, (N + s.B - 1) / s.B); }
static size_t packed_stats_bytes(const Shape& s, int N) {
  if (s.dtype != 1) return ((size_t)s.Hq * N * sizeof(float) + 255) / 256 * 256;
  return (size_t)s.Hq * win_packed_tiles(N, s.B + 1) * kTile * 32;
}
// Parts at most: as win_most_parts, but in fp32, where a query tile takes 6 us at d = 64 and 12 at
// 128, down to one each while the lists have a CU each or little more (a call for 1 sequence of
// 125, 32 heads of d = 128, 135 us with 8 tiles at least, 72 so; 20 of 5 to 100, 16 heads of d = 64,
// 121 and 66).
static int packed_most_parts(const Shape& s, int N) {
  const int T = packed_mean(s, N);
  const long all = (long)s.B * s.Hkv * ((T + kWinKeys - 1) / kWinKeys);
  const long every = ((long)T + kTile - 1) / kTile * (s.Hq / s.Hkv);
  const long least = s.dtype == 1 ? every / 8 : std::max(every / 8, std::min(every, 768 / all));
  return (int)std::max<long>(1, std::min<long>({16, 1024 / all, least}));
}
static size_t packed_sums_bytes(const Shape& s, int N, int parts) {
  return parts > 1 ? (size_t)parts * N * 2 * s.Hkv * s.D * sizeof(float) : 0;
}

// The cut, by win_cut's reasoning and numbers, for sequences half as long again as their mean
// (the longest lists are what a call waits for where there are few; the host knows only the
// mean).  (40 sequences of 1 to 511, window 255, 8 and 2 heads of d = 64: a call takes 66 us in
// one part of halves, 65, 59 and 56 in 2, 3 and 4 without; 40 of 255 48 and, in 4, 52; 16 of 1 to
// 2048, 16 and 4 heads of d = 128, 417 in one and 453 in 2.)
static WinParts packed_cut(const Shape& s, int N, int window) {
  const int G = s.Hq / s.Hkv, mean_len = packed_mean(s, N);
  const int T = (int)std::min<long>(N, (long)mean_len * 3 / 2);
  WinParts c = {};
  const double all = (N / (double)kWinKeys + (s.B - 1) / 2.0) * s.Hkv, every = std::ceil(T / 32.0);
  const double seen = std::min(every, std::ceil(((double)window + s.L + kWinKeys) / kTile) + 1);
  const double mean = seen - seen * seen / (2 * every);
  const bool f32 = s.dtype != 1;
  const double launch = 4.5, sum = (double)N * s.Hkv * s.D * (f32 ? 3.5e-6 : s.D == 128 ? 2.5e-6 : 1.25e-6);
  double best = 0;
  for (int h = f32 || s.D == 64 ? 1 : 2; h <= (f32 ? 1 : 2); ++h) {
    const double unit = f32 ? 6.0 * s.D / 64 : s.D == 128 ? 0.75 : h == 1 ? 0.65 : 0.4;
    const double fixed = f32 || s.D == 128 ? 6.0 : h == 1 ? 1.0 : 2.5;
    for (int p = 1; p <= packed_most_parts(s, N); ++p) {
      const double rounds = f32 || h == 2 ? std::ceil(all * p / 256) : std::max(1.0, all * p / 450);
      const double steps = f32 ? std::ceil(G * seen / p) : G * seen / p;  // (a step of fp32 is long)
      const double t = rounds * fixed + unit * steps * std::max(1.0, rounds * mean / seen) + (p > 1 ? launch + p * sum : 0);
      if (c.p == 0 || t < best) {
        best = t;
        c.p = p;
        c.halves = h == 2;
      }
    }
  }
  return c;
}

template <typename T, int D>
static hipError_t packed_backward_go(PackedArgs a, hipStream_t st) {
  const WinParts cut = packed_cut(a.s, a.N, a.window);
  a.sums = (float*)((char*)a.ws + packed_stats_bytes(a.s, a.N));
  win_backward_kernels<T, D>(a, cut, st);
  WindowArgs rows = a;  // as one sequence of all rows
  rows.s.B = 1;
  rows.T = a.N;
  return win_backward_sums<T, D>(rows, cut, cut.p > 1 ? a.N : 0, st);
}

hipError_t launch_packed_prefill(const PackedArgs& a_, hipStream_t st) {
  PackedArgs a = a_;
  a.T = packed_mean(a.s, a.N);
  if (a.s.dtype == 1) return a.s.D == 64 ? win_ring_go<64>(a, st) : win_ring_go<128>(a, st);
  return a.s.D == 64 ? win_prefill_f32_go<64>(a, st) : win_prefill_f32_go<128>(a, st);
}

hipError_t launch_packed_backward(const PackedArgs& a_, hipStream_t st) {
  PackedArgs a = a_;
  a.T = packed_mean(a.s, a.N);
  if (a.s.dtype == 1) return a.s.D == 64 ? packed_backward_go<bf16, 64>(a, st) : packed_backward_go<bf16, 128>(a, st);
  return a.s.D == 64 ? packed_backward_go<float, 64>(a, st) : packed_backward_go<float, 128>(a, st);
}

double packed_threads(const Shape& s, int N) {
  const double queries = (double)win_packed_queries(N, s.B + 1, s.Hq / s.Hkv, 2);
  const double keys = (double)win_packed_keys(N, s.B + 1) * packed_most_parts(s, N);
  return kWave * kWinWaves * 2.0 * s.Hkv * std::max(queries, keys);
}

size_t packed_backward_ws_bytes(const Shape& s, int N) {
  return packed_stats_bytes(s, N) + packed_sums_bytes(s, N, packed_most_parts(s, N));
}

// Threads of the largest launch (the grid's limit is checked by the caller): a
// workgroup of up to 512 threads per four units of queries, or per 128 keys and part,
// of which there are more than one in small grids only.
double window_threads(const Shape& s, int T) {
  const long units = ((long)T + kTile - 1) / kTile * (s.Hq / s.Hkv);
  const double queries = kWave * kWinWaves * 2 * (double)((units + kWinWaves - 1) / kWinWaves);
  const double keys = kWave * kWinWaves * 2 * std::ceil((double)T / kWinKeys);
  return (double)s.B * s.Hkv * std::max(queries, keys);
}

size_t window_backward_ws_bytes(const Shape& s, int T) {
  return win_stats_bytes(s, T) + win_sums_bytes(s, T);
}

}  // namespace hyb
