// api.cpp -- the C ABI of libhybattn: host-side validation, then dispatch to
// the kernel launchers.  Every check runs before any HIP call, so a rejected
// call enqueues nothing and touches no buffer.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/hybrid_attn.h"
#include "launch.h"
#include "launch_cache.h"
#include "launch_packed.h"

namespace {

thread_local std::string g_err;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

int ok() {
  g_err.clear();
  return HYB_OK;
}

size_t elem_bytes(int dtype) { return dtype == HYB_BF16 ? 2 : 4; }
size_t out_bytes(const hyb::Shape& s) { return s.out_f32 ? 4 : elem_bytes(s.dtype); }

// Shape checks common to every entry point.  need_state: the call reads a
// state pool.
int check_dims(const hyb_dims_t* d, bool need_state, hyb::Shape* s) {
  if (!d) return fail(HYB_ENULL, "dims is NULL");
  if (d->dtype != HYB_F32 && d->dtype != HYB_BF16)
    return fail(HYB_EDTYPE, "dtype %d is neither HYB_F32 nor HYB_BF16",
                d->dtype);
  if (d->batch < 0) return fail(HYB_EINVAL, "batch %d < 0", d->batch);
  if (d->n_q_heads < 1 || d->n_kv_heads < 1)
    return fail(HYB_EINVAL, "head counts must be >= 1 (Hq=%d, Hkv=%d)",
                d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads % d->n_kv_heads != 0)
    return fail(HYB_EINVAL, "n_kv_heads %d does not divide n_q_heads %d",
                d->n_kv_heads, d->n_q_heads);
  if (d->head_dim <= 0 || d->block <= 0 || d->feat_dim <= 0)
    return fail(HYB_EINVAL, "head_dim, block and feat_dim must be positive");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(HYB_EUNSUPPORTED, "head_dim %d not supported (64 or 128)",
                d->head_dim);
  if (d->feat_dim != 64 && d->feat_dim != 128 && d->feat_dim != 256)
    return fail(HYB_EUNSUPPORTED,
                "feat_dim %d not supported (64, 128 or 256)", d->feat_dim);
  if (d->block > 32)
    return fail(HYB_EUNSUPPORTED, "block %d not supported (1..32)", d->block);
  if (need_state && d->batch > 0 && d->n_slots < 1)
    return fail(HYB_EINVAL, "n_slots %d < 1", d->n_slots);
  if ((long long)d->batch * d->n_q_heads > 0x7fffffffLL)
    return fail(HYB_EINVAL, "batch * n_q_heads exceeds the grid limit");
  if (d->flags & ~(HYB_OUT_F32 | HYB_STEP_SPLIT | HYB_STEP_WHOLE | HYB_STEP_HALVES))
    return fail(HYB_EINVAL, "unknown flags 0x%x", d->flags);
  {
    const int kf = d->flags & (HYB_STEP_SPLIT | HYB_STEP_WHOLE | HYB_STEP_HALVES);
    if (kf & (kf - 1))
      return fail(HYB_EINVAL, "more than one of HYB_STEP_SPLIT, HYB_STEP_WHOLE, HYB_STEP_HALVES");
  }
  *s = hyb::Shape{d->batch,    d->n_q_heads,    d->n_kv_heads,
                  d->head_dim, d->block,        d->feat_dim / 2,
                  d->dtype,    d->n_slots,      (d->flags & HYB_OUT_F32) ? 1 : 0};
  s->step_kernel = (d->flags & HYB_STEP_SPLIT)    ? 1
                   : (d->flags & HYB_STEP_WHOLE)  ? 2
                   : (d->flags & HYB_STEP_HALVES) ? 3
                                                  : 0;
  if (s->step_kernel == 3 && !hyb::step_halves_supported(*s))
    return fail(HYB_EUNSUPPORTED,
                "HYB_STEP_HALVES needs bf16, feat_dim <= 128 and n_q_heads / n_kv_heads a "
                "multiple of 4");
  return HYB_OK;
}

// The step-kernel flags belong to hybrid_attn_step alone.
int no_step_flags(const hyb_dims_t* d) {
  if (d && (d->flags & (HYB_STEP_SPLIT | HYB_STEP_WHOLE | HYB_STEP_HALVES)))
    return fail(HYB_EINVAL,
                "HYB_STEP_SPLIT / HYB_STEP_WHOLE / HYB_STEP_HALVES apply to hybrid_attn_step only");
  return HYB_OK;
}

int check_ptr(const void* p, const char* name, bool required = true) {
  if (!p) return required ? fail(HYB_ENULL, "%s is NULL", name) : HYB_OK;
  if (reinterpret_cast<uintptr_t>(p) & 15)
    return fail(HYB_EALIGN, "%s is not 16-byte aligned", name);
  return HYB_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

int launched(hipError_t e, const char* what) {
  if (e != hipSuccess)
    return fail(HYB_ELAUNCH, "%s launch failed: %s", what,
                hipGetErrorString(e));
  return ok();
}

#define TRY(x)               \
  do {                       \
    int _rc = (x);           \
    if (_rc != HYB_OK) return _rc; \
  } while (0)

}  // namespace

extern "C" {

int hybrid_attn_step(const hyb_dims_t* dims, const void* q, const void* k,
                     const void* v, const void* W, const float* alpha,
                     const float* S, const float* z, const int32_t* slots,
                     const int32_t* block_len, void* out, void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, true, &s));
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(alpha, "alpha"));
  TRY(check_ptr(S, "S"));
  TRY(check_ptr(z, "z"));
  TRY(check_ptr(slots, "slots", false));
  TRY(check_ptr(block_len, "block_len", false));
  TRY(check_ptr(out, "out"));
  const size_t es = elem_bytes(s.dtype), f = 2 * (size_t)s.F;
  const size_t nq = (size_t)s.B * s.L * s.Hq * s.D * es;
  const size_t no = (size_t)s.B * s.L * s.Hq * s.D * out_bytes(s);
  const size_t nkv = (size_t)s.B * s.L * s.Hkv * s.D * es;
  const size_t nS = (size_t)s.n_slots * s.Hq * f * s.D * 4;
  const size_t nz = (size_t)s.n_slots * s.Hq * f * 4;
  const size_t nW = (size_t)s.Hq * s.F * s.D * es;
  if (overlap(out, no, q, nq) || overlap(out, no, k, nkv) ||
      overlap(out, no, v, nkv) || overlap(out, no, W, nW) ||
      overlap(out, no, S, nS) || overlap(out, no, z, nz) ||
      overlap(out, no, alpha, (size_t)s.Hq * 4) ||
      overlap(out, no, slots, (size_t)s.B * 4) ||
      overlap(out, no, block_len, (size_t)s.B * 4))
    return fail(HYB_EINVAL, "out overlaps an input");
  hyb::StepArgs a{s, q, k, v, W, alpha, S, z, slots, out, block_len};
  (void)hipGetLastError();
  return launched(hyb::launch_step(a, (hipStream_t)stream), "step");
}

int hybrid_attn_step_commit(const hyb_dims_t* dims, const void* q,
                            const void* k, const void* v, const void* W,
                            const float* alpha, float* S, float* z,
                            const int32_t* slots, const int32_t* block_len,
                            void* out, void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, true, &s));
  TRY(no_step_flags(dims));
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(alpha, "alpha"));
  TRY(check_ptr(S, "S"));
  TRY(check_ptr(z, "z"));
  TRY(check_ptr(slots, "slots", false));
  TRY(check_ptr(block_len, "block_len", false));
  TRY(check_ptr(out, "out"));
  const size_t es = elem_bytes(s.dtype), f = 2 * (size_t)s.F;
  const size_t nq = (size_t)s.B * s.L * s.Hq * s.D * es;
  const size_t no = (size_t)s.B * s.L * s.Hq * s.D * out_bytes(s);
  const size_t nkv = (size_t)s.B * s.L * s.Hkv * s.D * es;
  const size_t nS = (size_t)s.n_slots * s.Hq * f * s.D * 4;
  const size_t nz = (size_t)s.n_slots * s.Hq * f * 4;
  const size_t nW = (size_t)s.Hq * s.F * s.D * es;
  // Everything the kernel writes (out, S, z) is disjoint from everything it
  // reads and from each other.
  struct Buf {
    const void* p;
    size_t n;
  };
  const Buf written[3] = {{out, no}, {S, nS}, {z, nz}};
  const Buf read_only[7] = {{q, nq},     {k, nkv},
                            {v, nkv},     {W, nW},
                            {alpha, (size_t)s.Hq * 4}, {slots, (size_t)s.B * 4},
                            {block_len, (size_t)s.B * 4}};
  for (int i = 0; i < 3; ++i) {
    for (const Buf& r : read_only)
      if (overlap(written[i].p, written[i].n, r.p, r.n))
        return fail(HYB_EINVAL, "an output (out, S or z) overlaps an input");
    for (int j = i + 1; j < 3; ++j)
      if (overlap(written[i].p, written[i].n, written[j].p, written[j].n))
        return fail(HYB_EINVAL, "out, S and z overlap");
  }
  hyb::StepArgs a{s, q, k, v, W, alpha, S, z, slots, out, block_len};
  (void)hipGetLastError();
  return launched(hyb::launch_step_commit(a, (hipStream_t)stream), "step_commit");
}

int hybrid_state_commit(const hyb_dims_t* dims, const void* k, const void* v,
                        const void* W, float* S, float* z,
                        const int32_t* slots, const int32_t* block_len,
                        void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, true, &s));
  TRY(no_step_flags(dims));
  if (s.B == 0) return ok();
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(S, "S"));
  TRY(check_ptr(z, "z"));
  TRY(check_ptr(slots, "slots", false));
  TRY(check_ptr(block_len, "block_len", false));
  const size_t f = 2 * (size_t)s.F;
  const size_t nS = (size_t)s.n_slots * s.Hq * f * s.D * 4;
  const size_t nz = (size_t)s.n_slots * s.Hq * f * 4;
  if (overlap(S, nS, z, nz)) return fail(HYB_EINVAL, "S and z overlap");
  hyb::CommitArgs a{s, k, v, W, S, z, slots, block_len};
  (void)hipGetLastError();
  return launched(hyb::launch_commit(a, (hipStream_t)stream), "commit");
}

}  // extern "C"

namespace {

// Validation and dispatch of the prefill.  ws == nullptr with use_scratch:
// the workspace is the library-held scratch buffer.
int prefill_impl(const hyb_dims_t* dims, int32_t seq_len, const void* q,
                 const void* k, const void* v, const void* W,
                 const float* alpha, float* S, float* z, const int32_t* slots,
                 void* out, void* ws, size_t ws_bytes, bool use_scratch,
                 void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, true, &s));
  TRY(no_step_flags(dims));
  if (seq_len <= 0 || seq_len % s.L != 0)
    return fail(HYB_EINVAL, "seq_len %d is not a positive multiple of block %d",
                seq_len, s.L);
  if (s.B == 0) return ok();
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(S, "S"));
  TRY(check_ptr(z, "z"));
  TRY(check_ptr(slots, "slots", false));
  TRY(check_ptr(out, "out", false));
  if (out) {
    TRY(check_ptr(q, "q"));
    TRY(check_ptr(alpha, "alpha"));
  }
  const size_t need = hybrid_workspace_bytes(dims, HYB_OP_PREFILL, seq_len);
  if (use_scratch) {
    if (need > hyb::kScratchBytes)
      return fail(HYB_EWORKSPACE,
                  "prefill needs %zu scratch bytes, more than the %zu "
                  "(HYB_NOALLOC_SCRATCH_BYTES) the library holds; use "
                  "hybrid_state_prefill with a workspace",
                  need, hyb::kScratchBytes);
  } else {
    if (need > 0 && (!ws || ws_bytes < need))
      return fail(HYB_EWORKSPACE, "prefill needs %zu workspace bytes, got %zu",
                  need, ws ? ws_bytes : (size_t)0);
    TRY(check_ptr(ws, "ws", false));
  }
  const size_t es = elem_bytes(s.dtype), f = 2 * (size_t)s.F;
  const size_t nq = (size_t)s.B * seq_len * s.Hq * s.D * es;
  const size_t no = (size_t)s.B * seq_len * s.Hq * s.D * out_bytes(s);
  const size_t nkv = (size_t)s.B * seq_len * s.Hkv * s.D * es;
  const size_t nS = (size_t)s.n_slots * s.Hq * f * s.D * 4;
  const size_t nz = (size_t)s.n_slots * s.Hq * f * 4;
  if (overlap(S, nS, z, nz)) return fail(HYB_EINVAL, "S and z overlap");
  if (out && (overlap(out, no, q, nq) || overlap(out, no, k, nkv) ||
              overlap(out, no, v, nkv) || overlap(out, no, S, nS) ||
              overlap(out, no, z, nz)))
    return fail(HYB_EINVAL, "out overlaps an input");
  if (need > 0 && (overlap(ws, need, S, nS) || overlap(ws, need, z, nz) ||
                   overlap(ws, need, k, nkv) || overlap(ws, need, v, nkv) ||
                   (out && (overlap(ws, need, out, no) || overlap(ws, need, q, nq)))))
    return fail(HYB_EINVAL, "the workspace overlaps an argument");
  (void)hipGetLastError();
  if (use_scratch && need > 0) {
    void* p = nullptr;
    const hipError_t e = hyb::scratch_device_ptr(&p);
    if (e != hipSuccess)
      return fail(HYB_ELAUNCH, "scratch buffer lookup failed: %s",
                  hipGetErrorString(e));
    ws = p;
  }
  hyb::PrefillArgs a{s, seq_len, q, k, v, W, alpha, S, z, slots, out, (float*)ws};
  return launched(hyb::launch_prefill(a, (hipStream_t)stream), "prefill");
}

}  // namespace

extern "C" {

int hybrid_state_prefill(const hyb_dims_t* dims, int32_t seq_len,
                         const void* q, const void* k, const void* v,
                         const void* W, const float* alpha, float* S, float* z,
                         const int32_t* slots, void* out, void* ws,
                         size_t ws_bytes, void* stream) {
  return prefill_impl(dims, seq_len, q, k, v, W, alpha, S, z, slots, out, ws,
                      ws_bytes, false, stream);
}

int hybrid_state_prefill_noalloc(const hyb_dims_t* dims, int32_t seq_len,
                                 const void* q, const void* k, const void* v,
                                 const void* W, const float* alpha, float* S,
                                 float* z, const int32_t* slots, void* out,
                                 void* stream) {
  return prefill_impl(dims, seq_len, q, k, v, W, alpha, S, z, slots, out,
                      nullptr, 0, true, stream);
}

}  // extern "C"

namespace {

// Validation and dispatch of the softmax-prefix step; !paged:
// contiguous cache [B][max_prefix][Hkv][d]; otherwise page pools
// [n_pages][page_size][Hkv][d] and a [B][max_pages] page table.
int softmax_prefix_impl(const hyb_dims_t* dims, const void* q, const void* k,
                        const void* v, const void* k_cache,
                        const void* v_cache, const int32_t* prefix_len,
                        int32_t max_prefix, bool paged,
                        const int32_t* page_table, int32_t n_pages,
                        int32_t page_size, int32_t max_pages, void* out,
                        void* ws, size_t ws_bytes, void* stream,
                        int32_t window = -1, int32_t n_sinks = 0,
                        const int32_t* block_len = nullptr) {
  hyb::Shape s;
  const bool win = window >= 0;  // (paged only)
  const char* name = win ? "softmax_window_step_paged" : "softmax_prefix_step";
  TRY(check_dims(dims, false, &s));
  TRY(no_step_flags(dims));
  int page_shift = 0;
  if (paged) {
    if (max_pages < 0) return fail(HYB_EINVAL, "max_pages %d < 0", max_pages);
    if (page_size < 32 || page_size > (1 << 16) || (page_size & (page_size - 1)))
      return fail(HYB_EUNSUPPORTED,
                  "page_size %d not supported (a power of two, 32 .. 65536)",
                  page_size);
    while ((1 << page_shift) < page_size) ++page_shift;
    if ((long long)max_pages * page_size > 0x7fffffffLL - 64)
      return fail(HYB_EINVAL, "max_pages * page_size exceeds the index range");
    if (max_pages > 0 && n_pages < 1)
      return fail(HYB_EINVAL, "n_pages %d < 1", n_pages);
    max_prefix = max_pages * page_size;
  }
  if (max_prefix < 0)
    return fail(HYB_EINVAL, "max_prefix %d < 0", max_prefix);
  if (s.Hq / s.Hkv > 8)
    return fail(HYB_EUNSUPPORTED,
                "%s supports up to 8 query heads per KV head", name);
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(prefix_len, "prefix_len"));
  if (max_prefix > 0) {
    TRY(check_ptr(k_cache, paged ? "k_pages" : "k_cache"));
    TRY(check_ptr(v_cache, paged ? "v_pages" : "v_cache"));
    if (paged) TRY(check_ptr(page_table, "page_table"));
  }
  TRY(check_ptr(block_len, "block_len", false));
  // cached tokens that a query sees, at most (a window's ends share tiles with
  // hidden tokens)
  const int max_seen =
      win ? (int)std::min<long long>(max_prefix, (long long)window + n_sinks + 64) : max_prefix;
  const size_t need =
      hybrid_workspace_bytes(dims, win ? HYB_OP_WINDOW_STEP : HYB_OP_SOFTMAX_PREFIX, max_seen);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(HYB_EWORKSPACE, "%s needs %zu workspace bytes, got %zu", name,
                need, ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws", false));
  const size_t es = elem_bytes(s.dtype);
  const size_t nq = (size_t)s.B * s.L * s.Hq * s.D * es;
  const size_t no = (size_t)s.B * s.L * s.Hq * s.D * out_bytes(s);
  const size_t nkv = (size_t)s.B * s.L * s.Hkv * s.D * es;
  const size_t nc = paged ? (size_t)n_pages * page_size * s.Hkv * s.D * es
                          : (size_t)s.B * max_prefix * s.Hkv * s.D * es;
  const size_t nt = paged ? (size_t)s.B * max_pages * 4 : 0;
  if (overlap(out, no, q, nq) || overlap(out, no, k, nkv) ||
      overlap(out, no, v, nkv) || overlap(out, no, k_cache, nc) ||
      overlap(out, no, v_cache, nc) || overlap(out, no, ws, need) ||
      overlap(out, no, prefix_len, (size_t)s.B * 4) ||
      overlap(out, no, block_len, (size_t)s.B * 4) ||
      overlap(out, no, page_table, nt))
    return fail(HYB_EINVAL, "out overlaps an input or the workspace");
  // the split kernels write the workspace while they read the inputs
  if (need > 0 && (overlap(ws, need, q, nq) || overlap(ws, need, k, nkv) ||
                   overlap(ws, need, v, nkv) || overlap(ws, need, k_cache, nc) ||
                   overlap(ws, need, v_cache, nc) ||
                   overlap(ws, need, prefix_len, (size_t)s.B * 4) ||
                   overlap(ws, need, block_len, (size_t)s.B * 4) ||
                   overlap(ws, need, page_table, nt)))
    return fail(HYB_EINVAL, "the workspace overlaps an input");
  hyb::SoftmaxPrefixArgs a{s,         q,   k,  v,
                           k_cache,   v_cache, prefix_len, max_prefix,
                           out,       ws,
                           win ? hyb::softmax_window_splits(s, max_seen) : hyb::softmax_prefix_splits(s, max_seen),
                           paged && max_prefix > 0 ? page_table : nullptr,
                           page_shift, max_pages, n_pages, max_seen,
                           window,    n_sinks, block_len};
  (void)hipGetLastError();
  return launched(hyb::launch_softmax_prefix(a, (hipStream_t)stream), name);
}

}  // namespace

extern "C" {

int softmax_prefix_step(const hyb_dims_t* dims, const void* q, const void* k,
                        const void* v, const void* k_cache,
                        const void* v_cache, const int32_t* prefix_len,
                        int32_t max_prefix, void* out, void* ws,
                        size_t ws_bytes, void* stream) {
  return softmax_prefix_impl(dims, q, k, v, k_cache, v_cache, prefix_len,
                             max_prefix, false, nullptr, 0, 0, 0, out, ws,
                             ws_bytes, stream);
}

int softmax_prefix_step_paged(const hyb_dims_t* dims, const void* q,
                              const void* k, const void* v,
                              const void* k_pages, const void* v_pages,
                              int32_t n_pages, int32_t page_size,
                              const int32_t* page_table, int32_t max_pages,
                              const int32_t* prefix_len, void* out, void* ws,
                              size_t ws_bytes, void* stream) {
  return softmax_prefix_impl(dims, q, k, v, k_pages, v_pages, prefix_len, 0,
                             true, page_table, n_pages, page_size, max_pages,
                             out, ws, ws_bytes, stream);
}

int softmax_window_step_paged(const hyb_dims_t* dims, const void* q,
                              const void* k, const void* v,
                              const void* k_pages, const void* v_pages,
                              int32_t n_pages, int32_t page_size,
                              const int32_t* page_table, int32_t max_pages,
                              const int32_t* prefix_len, int32_t window,
                              int32_t n_sinks, const int32_t* block_len,
                              void* out, void* ws, size_t ws_bytes,
                              void* stream) {
  if (window < 0 || n_sinks < 0)
    return fail(HYB_EINVAL, "window %d and n_sinks %d must be >= 0", window, n_sinks);
  if (dims && dims->n_q_heads > 65536)
    return fail(HYB_EUNSUPPORTED, "n_q_heads %d not supported (at most 65536)", dims->n_q_heads);
  return softmax_prefix_impl(dims, q, k, v, k_pages, v_pages, prefix_len, 0,
                             true, page_table, n_pages, page_size, max_pages,
                             out, ws, ws_bytes, stream, window, n_sinks, block_len);
}

}  // extern "C"

namespace {

struct Buf {
  const void* p;
  size_t n;
};

// Outputs (with the workspace) must not overlap each other or an input.
int check_overlaps(const Buf* written, int nw, const Buf* read_only, int nr) {
  for (int i = 0; i < nw; ++i) {
    for (int j = i + 1; j < nw; ++j)
      if (overlap(written[i].p, written[i].n, written[j].p, written[j].n))
        return fail(HYB_EINVAL, "outputs or the workspace overlap each other");
    for (int j = 0; j < nr; ++j)
      if (overlap(written[i].p, written[i].n, read_only[j].p, read_only[j].n))
        return fail(HYB_EINVAL, "an output or the workspace overlaps an input");
  }
  return HYB_OK;
}

// What softmax_window_prefill and its gradient check alike.
int check_window(const hyb_dims_t* dims, int32_t seq_len, int32_t window,
                 int32_t n_sinks, hyb::Shape* s) {
  TRY(check_dims(dims, false, s));
  TRY(no_step_flags(dims));
  if (seq_len <= 0 || seq_len > (1 << 30))
    return fail(HYB_EINVAL, "seq_len %d is not in 1 .. 2^30", seq_len);
  if (window < 0 || n_sinks < 0)
    return fail(HYB_EINVAL, "window %d and n_sinks %d must be >= 0", window, n_sinks);
  if (s->Hq > 65536) return fail(HYB_EUNSUPPORTED, "n_q_heads %d not supported (at most 65536)", s->Hq);
  if (hyb::window_threads(*s, seq_len) > 0xffffffffL)
    return fail(HYB_EINVAL, "batch * heads * seq_len exceeds the grid limit");
  return HYB_OK;
}

}  // namespace

extern "C" {

int softmax_window_prefill(const hyb_dims_t* dims, int32_t seq_len,
                           int32_t window, int32_t n_sinks, const void* q,
                           const void* k, const void* v,
                           const int32_t* seq_lens, void* out, float* lse,
                           void* ws, size_t ws_bytes, void* stream) {
  hyb::Shape s;
  TRY(check_window(dims, seq_len, window, n_sinks, &s));
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(seq_lens, "seq_lens", false));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(lse, "lse", false));
  const size_t need = hybrid_workspace_bytes(dims, HYB_OP_WINDOW_PREFILL, seq_len);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(HYB_EWORKSPACE, "softmax_window_prefill needs %zu workspace bytes, got %zu",
                need, ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws", false));
  const size_t rows = (size_t)s.B * seq_len, es = elem_bytes(s.dtype);
  const Buf written[] = {{out, rows * s.Hq * s.D * out_bytes(s)}, {lse, rows * s.Hq * 4}, {ws, need}};
  const Buf read_only[] = {{q, rows * s.Hq * s.D * es},
                           {k, rows * s.Hkv * s.D * es},
                           {v, rows * s.Hkv * s.D * es},
                           {seq_lens, (size_t)s.B * 4}};
  TRY(check_overlaps(written, 3, read_only, 4));
  hyb::WindowArgs a{s, seq_len, window, n_sinks, q, k, v, seq_lens, out, lse};
  (void)hipGetLastError();
  return launched(hyb::launch_window_prefill(a, (hipStream_t)stream), "softmax_window_prefill");
}

int softmax_window_backward(const hyb_dims_t* dims, int32_t seq_len,
                            int32_t window, int32_t n_sinks, const void* q,
                            const void* k, const void* v,
                            const int32_t* seq_lens, const void* out,
                            const float* lse, const void* dout, void* dq,
                            void* dk, void* dv, void* ws, size_t ws_bytes,
                            void* stream) {
  hyb::Shape s;
  TRY(check_window(dims, seq_len, window, n_sinks, &s));
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(seq_lens, "seq_lens", false));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(lse, "lse"));
  TRY(check_ptr(dout, "dout"));
  TRY(check_ptr(dq, "dq"));
  TRY(check_ptr(dk, "dk"));
  TRY(check_ptr(dv, "dv"));
  const size_t need = hybrid_workspace_bytes(dims, HYB_OP_WINDOW_BACKWARD, seq_len);
  if (!ws || ws_bytes < need)
    return fail(HYB_EWORKSPACE, "softmax_window_backward needs %zu workspace bytes, got %zu",
                need, ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws"));
  const size_t rows = (size_t)s.B * seq_len, es = elem_bytes(s.dtype);
  const size_t nq = rows * s.Hq * s.D, nkv = rows * s.Hkv * s.D;
  const Buf written[] = {{dq, nq * out_bytes(s)}, {dk, nkv * out_bytes(s)}, {dv, nkv * out_bytes(s)}, {ws, need}};
  const Buf read_only[] = {{q, nq * es},   {k, nkv * es},    {v, nkv * es},  {seq_lens, (size_t)s.B * 4},
                           {out, nq * es}, {dout, nq * es}, {lse, rows * s.Hq * 4}};
  TRY(check_overlaps(written, 4, read_only, 7));
  // (out and lse are only read)
  hyb::WindowArgs a{s, seq_len, window, n_sinks, q, k, v, seq_lens,
                    const_cast<void*>(out), const_cast<float*>(lse), dout, dq, dk, dv, (float*)ws};
  (void)hipGetLastError();
  return launched(hyb::launch_window_backward(a, (hipStream_t)stream), "softmax_window_backward");
}

}  // extern "C"

namespace {

// Rows of n bytes at p, `stride` bytes apart.
struct Rows {
  const void* p;
  size_t n, stride;
};
bool rows_overlap(const Rows& a, const Rows& b, long count) {
  if (!a.p || !b.p || count == 0) return false;
  const size_t na = (count - 1) * a.stride + a.n, nb = (count - 1) * b.stride + b.n;
  if (!overlap(a.p, na, b.p, nb)) return false;
  if (count == 1 || a.stride != b.stride) return true;
  // the same stride: where b's rows fall between a's
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  const size_t d = y >= x ? (y - x) % a.stride : (a.stride - (x - y) % a.stride) % a.stride;
  return d < a.n || d + b.n > a.stride;
}

int check_rope(const hyb_rope_dims_t* d, hyb::RopeArgs* a) {
  if (!d) return fail(HYB_ENULL, "dims is NULL");
  if ((d->dtype != HYB_F32 && d->dtype != HYB_BF16) || (d->grad_dtype != HYB_F32 && d->grad_dtype != HYB_BF16))
    return fail(HYB_EDTYPE, "dtype %d or grad_dtype %d is neither HYB_F32 nor HYB_BF16", d->dtype, d->grad_dtype);
  if (d->tokens < 0) return fail(HYB_EINVAL, "tokens %d < 0", d->tokens);
  if (d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads > (1 << 20) || d->n_kv_heads > (1 << 20))
    return fail(HYB_EINVAL, "head counts must be 1 .. 2^20 (Hq=%d, Hkv=%d)", d->n_q_heads, d->n_kv_heads);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(HYB_EUNSUPPORTED, "head_dim %d not supported (64 or 128)", d->head_dim);
  if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 8)
    return fail(HYB_EUNSUPPORTED, "rot_dim %d not supported (a multiple of 8, 0 .. head_dim)", d->rot_dim);
  if (d->layout != HYB_ROPE_HALF && d->layout != HYB_ROPE_INTERLEAVED)
    return fail(HYB_EINVAL, "unknown layout %d", d->layout);
  if (d->flags & ~HYB_OUT_F32) return fail(HYB_EINVAL, "unknown flags 0x%x", d->flags);
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps) || !std::isfinite(d->rot_scale))
    return fail(HYB_EINVAL, "eps must be positive and finite, rot_scale finite");
  const long nq = (long)d->n_q_heads * d->head_dim, nk = (long)d->n_kv_heads * d->head_dim;
  const long given[5] = {d->q_stride, d->k_stride, d->v_stride, d->q_out_stride, d->k_out_stride};
  const long least[5] = {nq, nk, nk, nq, nk};
  long* set[5] = {&a->q_stride, &a->k_stride, &a->v_stride, &a->q_out_stride, &a->k_out_stride};
  for (int i = 0; i < 5; ++i) {
    if (given[i] != 0 && (given[i] < least[i] || given[i] > (1L << 31)))
      return fail(HYB_EINVAL, "a row stride of %ld is shorter than the row, or longer than 2^31", given[i]);
    if (given[i] % 8) return fail(HYB_EALIGN, "a row stride of %ld is not a multiple of 8 elements", given[i]);
    *set[i] = given[i] ? given[i] : least[i];
  }
  a->N = d->tokens;
  a->Hq = d->n_q_heads;
  a->Hkv = d->n_kv_heads;
  a->D = d->head_dim;
  a->rot = d->rot_dim;
  a->interleaved = d->layout == HYB_ROPE_INTERLEAVED;
  a->dtype = d->dtype;
  a->grad_dtype = d->grad_dtype;
  a->out_f32 = d->dtype == HYB_F32 || (d->flags & HYB_OUT_F32);
  a->eps = d->eps;
  a->rot_scale = d->rot_scale;
  return HYB_OK;
}

// Written rows must not overlap each other or anything that is read.
int check_rows(const Rows* written, int nw, const Rows* read_only, int nr, long count) {
  for (int i = 0; i < nw; ++i) {
    for (int j = i + 1; j < nw; ++j)
      if (rows_overlap(written[i], written[j], count))
        return fail(HYB_EINVAL, "the outputs overlap each other");
    for (int j = 0; j < nr; ++j)
      if (rows_overlap(written[i], read_only[j], count))
        return fail(HYB_EINVAL, "an output overlaps an input");
  }
  return HYB_OK;
}

// Whole buffers against each other and against rows.
int check_buffers(const Buf* bufs, int n, bool written, const Rows* rows, int nr, long count) {
  for (int i = 0; i < n; ++i) {
    for (int j = i + 1; written && j < n; ++j)
      if (overlap(bufs[i].p, bufs[i].n, bufs[j].p, bufs[j].n))
        return fail(HYB_EINVAL, "outputs or the workspace overlap each other");
    for (int j = 0; j < nr; ++j)
      if (rows[j].p && overlap(bufs[i].p, bufs[i].n, rows[j].p, (count - 1) * rows[j].stride + rows[j].n))
        return fail(HYB_EINVAL, "an output or the workspace overlaps another argument");
  }
  return HYB_OK;
}

int rope_impl(const hyb_rope_dims_t* dims, const void* q, const void* k,
              const void* v, const void* wq, const void* wk,
              const int32_t* positions, const double* inv_freq,
              const int32_t* slots, void* q_out, void* k_out, void* k_pages,
              void* v_pages, int32_t n_pages, int32_t page_size, bool paged,
              void* stream) {
  hyb::RopeArgs a{};
  TRY(check_rope(dims, &a));
  if (paged && (n_pages < 1 || page_size < 1))
    return fail(HYB_EINVAL, "n_pages %d and page_size %d must be >= 1", n_pages, page_size);
  if (a.N == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(wq, "wq", false));
  TRY(check_ptr(wk, "wk", false));
  TRY(check_ptr(positions, "positions"));
  TRY(check_ptr(inv_freq, "inv_freq", a.rot > 0));
  TRY(check_ptr(q_out, "q_out"));
  TRY(check_ptr(k_out, "k_out", !paged));
  if (paged) {
    TRY(check_ptr(v, "v"));
    TRY(check_ptr(slots, "slots"));
    TRY(check_ptr(k_pages, "k_pages"));
    TRY(check_ptr(v_pages, "v_pages"));
  }
  const size_t es = elem_bytes(a.dtype), eo = a.out_f32 ? 4 : es;
  const size_t nq = (size_t)a.Hq * a.D, nk = (size_t)a.Hkv * a.D;
  const Rows outs[2] = {{q_out, nq * eo, a.q_out_stride * eo}, {k_out, nk * eo, a.k_out_stride * eo}};
  const Rows ins[3] = {{q, nq * es, a.q_stride * es}, {k, nk * es, a.k_stride * es}, {v, nk * es, a.v_stride * es}};
  TRY(check_rows(outs, 2, ins, 3, a.N));
  const Buf small[] = {{wq, a.D * es}, {wk, a.D * es}, {positions, (size_t)a.N * 4},
                       {inv_freq, (size_t)a.rot * 4}, {slots, (size_t)a.N * 4}};
  TRY(check_buffers(small, 5, false, outs, 2, a.N));
  if (paged) {
    a.n_rows = (long)n_pages * page_size;
    const Buf pools[2] = {{k_pages, a.n_rows * nk * es}, {v_pages, a.n_rows * nk * es}};
    TRY(check_buffers(pools, 2, true, outs, 2, a.N));
    TRY(check_buffers(pools, 2, true, ins, 3, a.N));
    TRY(check_overlaps(pools, 2, small, 5));
  }
  a.q = q, a.k = k, a.v = v, a.wq = wq, a.wk = wk;
  a.positions = positions, a.inv_freq = inv_freq;
  a.q_out = q_out, a.k_out = k_out;
  a.slots = slots, a.k_pages = k_pages, a.v_pages = v_pages;
  (void)hipGetLastError();
  return launched(hyb::launch_rope(a, (hipStream_t)stream), paged ? "qk_norm_rope_paged" : "qk_norm_rope");
}

}  // namespace

extern "C" {

int hybrid_qk_norm_rope(const hyb_rope_dims_t* dims, const void* q,
                        const void* k, const void* wq, const void* wk,
                        const int32_t* positions, const double* inv_freq,
                        void* q_out, void* k_out, void* stream) {
  return rope_impl(dims, q, k, nullptr, wq, wk, positions, inv_freq, nullptr, q_out, k_out, nullptr, nullptr, 0, 0,
                   false, stream);
}

int hybrid_qk_norm_rope_paged(const hyb_rope_dims_t* dims, const void* q,
                              const void* k, const void* v, const void* wq,
                              const void* wk, const int32_t* positions,
                              const double* inv_freq, const int32_t* slots,
                              void* q_out, void* k_out, void* k_pages,
                              void* v_pages, int32_t n_pages,
                              int32_t page_size, void* stream) {
  return rope_impl(dims, q, k, v, wq, wk, positions, inv_freq, slots, q_out, k_out, k_pages, v_pages, n_pages,
                   page_size, true, stream);
}

size_t hybrid_rope_workspace_bytes(const hyb_rope_dims_t* dims) {
  hyb::RopeArgs a{};
  const std::string saved = g_err;
  const int rc = check_rope(dims, &a);
  g_err = saved;
  return rc == HYB_OK ? hyb::rope_backward_ws_bytes(a) : 0;
}

int hybrid_qk_norm_rope_backward(const hyb_rope_dims_t* dims, const void* q,
                                 const void* k, const void* wq, const void* wk,
                                 const int32_t* positions,
                                 const double* inv_freq, const void* dq_out,
                                 const void* dk_out, void* dq, void* dk,
                                 float* dwq, float* dwk, void* ws,
                                 size_t ws_bytes, void* stream) {
  hyb::RopeArgs a{};
  TRY(check_rope(dims, &a));
  TRY(check_ptr(wq, "wq", false));
  TRY(check_ptr(wk, "wk", false));
  if ((wq != nullptr) != (dwq != nullptr) || (wk != nullptr) != (dwk != nullptr))
    return fail(HYB_ENULL, "dwq and dwk are required exactly where wq and wk are given");
  TRY(check_ptr(dwq, "dwq", false));
  TRY(check_ptr(dwk, "dwk", false));
  const bool none = a.N == 0;
  if (none && !dwq && !dwk) return ok();
  TRY(check_ptr(q, "q", !none));
  TRY(check_ptr(k, "k", !none));
  TRY(check_ptr(positions, "positions", !none));
  TRY(check_ptr(inv_freq, "inv_freq", !none && a.rot > 0));
  TRY(check_ptr(dq_out, "dq_out", !none));
  TRY(check_ptr(dk_out, "dk_out", !none));
  TRY(check_ptr(dq, "dq", !none));
  TRY(check_ptr(dk, "dk", !none));
  const size_t need = wq || wk ? hyb::rope_backward_ws_bytes(a) : 0;
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(HYB_EWORKSPACE, "qk_norm_rope_backward needs %zu workspace bytes, got %zu", need,
                ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws", false));
  const size_t es = elem_bytes(a.dtype), eo = a.out_f32 ? 4 : es, eg = elem_bytes(a.grad_dtype);
  const size_t nq = (size_t)a.Hq * a.D, nk = (size_t)a.Hkv * a.D;
  const Rows outs[2] = {{dq, nq * eo, a.q_out_stride * eo}, {dk, nk * eo, a.k_out_stride * eo}};
  const Rows ins[4] = {{q, nq * es, a.q_stride * es}, {k, nk * es, a.k_stride * es},
                       {dq_out, nq * eg, nq * eg}, {dk_out, nk * eg, nk * eg}};
  const Buf sums[3] = {{dwq, (size_t)a.D * 4}, {dwk, (size_t)a.D * 4}, {ws, need}};
  const Buf small[4] = {{wq, a.D * es}, {wk, a.D * es}, {positions, (size_t)a.N * 4}, {inv_freq, (size_t)a.rot * 4}};
  TRY(check_overlaps(sums, 3, small, 4));
  if (!none) {
    TRY(check_rows(outs, 2, ins, 4, a.N));
    TRY(check_buffers(small, 4, false, outs, 2, a.N));
    TRY(check_buffers(sums, 3, true, outs, 2, a.N));
    TRY(check_buffers(sums, 3, true, ins, 4, a.N));
  }
  a.q = q, a.k = k, a.wq = wq, a.wk = wk;
  a.positions = positions, a.inv_freq = inv_freq;
  a.dq_out = dq_out, a.dk_out = dk_out, a.dq = dq, a.dk = dk;
  a.dwq = dwq, a.dwk = dwk;
  a.ws = need > 0 ? (float*)ws : nullptr;
  (void)hipGetLastError();
  return launched(hyb::launch_rope_backward(a, (hipStream_t)stream), "qk_norm_rope_backward");
}

int kv_pages_plan(int32_t batch, int32_t max_pages, int32_t page_size,
                  int32_t n_free, int32_t max_tokens,
                  const int32_t* prefix_len, const int32_t* new_len,
                  const int32_t* free_pages, int32_t* page_table,
                  int32_t* slots, int32_t* positions, int32_t* token_start,
                  int32_t* counts, void* stream) {
  if (batch < 0 || max_pages < 0 || n_free < 0 || max_tokens < 0)
    return fail(HYB_EINVAL, "batch %d, max_pages %d, n_free %d and max_tokens %d must be >= 0", batch, max_pages,
                n_free, max_tokens);
  if (batch > hyb::kMaxPlanBatch)
    return fail(HYB_EUNSUPPORTED, "batch %d not supported (at most %d)", batch, hyb::kMaxPlanBatch);
  if (page_size < 1 || page_size > (1 << 16) || (page_size & (page_size - 1)))
    return fail(HYB_EUNSUPPORTED, "page_size %d not supported (a power of two, 1 .. 65536)", page_size);
  if ((long long)max_pages * page_size > 0x7fffffffLL - 64)
    return fail(HYB_EINVAL, "max_pages * page_size exceeds the index range");
  if (batch == 0) return ok();
  TRY(check_ptr(prefix_len, "prefix_len"));
  TRY(check_ptr(new_len, "new_len"));
  if (!free_pages && n_free > 0) return fail(HYB_ENULL, "free_pages is NULL");
  if (reinterpret_cast<uintptr_t>(free_pages) & 3) return fail(HYB_EALIGN, "free_pages is not 4-byte aligned");
  TRY(check_ptr(page_table, "page_table", max_pages > 0));
  TRY(check_ptr(slots, "slots", max_tokens > 0));
  TRY(check_ptr(positions, "positions", max_tokens > 0));
  TRY(check_ptr(token_start, "token_start"));
  TRY(check_ptr(counts, "counts"));
  const Buf written[] = {{page_table, (size_t)batch * max_pages * 4}, {slots, (size_t)max_tokens * 4},
                         {positions, (size_t)max_tokens * 4}, {token_start, (size_t)(batch + 1) * 4}, {counts, 8}};
  const Buf read_only[] = {{prefix_len, (size_t)batch * 4}, {new_len, (size_t)batch * 4},
                           {free_pages, (size_t)n_free * 4}};
  TRY(check_overlaps(written, 5, read_only, 3));
  int shift = 0;
  while ((1 << shift) < page_size) ++shift;
  hyb::PagesArgs a{batch, max_pages, shift, n_free, max_tokens, prefix_len, new_len, free_pages,
                   page_table, slots, positions, token_start, counts};
  (void)hipGetLastError();
  return launched(hyb::launch_pages_plan(a, (hipStream_t)stream), "kv_pages_plan");
}

}  // extern "C"

namespace {

int check_page(int32_t page_size, int32_t scale_block, int32_t max_pages, int32_t n_pages, int* page_shift, int* sb_shift) {
  if (max_pages < 0) return fail(HYB_EINVAL, "max_pages %d < 0", max_pages);
  if (page_size < 32 || page_size > (1 << 16) || (page_size & (page_size - 1)))
    return fail(HYB_EUNSUPPORTED, "page_size %d not supported (a power of two, 32 .. 65536)", page_size);
  if (scale_block < 32 || scale_block > page_size || (scale_block & (scale_block - 1)))
    return fail(HYB_EUNSUPPORTED, "scale_block %d not supported (a power of two, 32 .. page_size)", scale_block);
  if ((long long)max_pages * page_size > 0x7fffffffLL - 64)
    return fail(HYB_EINVAL, "max_pages * page_size exceeds the index range");
  if (max_pages > 0 && n_pages < 1) return fail(HYB_EINVAL, "n_pages %d < 1", n_pages);
  for (*page_shift = 0; (1 << *page_shift) < page_size;) ++*page_shift;
  for (*sb_shift = 0; (1 << *sb_shift) < scale_block;) ++*sb_shift;
  return HYB_OK;
}

// Validation and dispatch of the 8-bit cache's write, and (read) of its reverse.
int kv_q8_impl(const hyb_kv_q8_dims_t* d, const void* k, const void* v, const void* k_pages, const void* v_pages,
               const uint8_t* k_scales, const uint8_t* v_scales, const int32_t* page_table, const int32_t* first,
               const int32_t* token_start, bool read, void* stream) {
  const char* name = read ? "kv_pages_q8_read" : "kv_pages_q8_write";
  if (!d) return fail(HYB_ENULL, "dims is NULL");
  if (d->dtype != HYB_F32 && d->dtype != HYB_BF16)
    return fail(HYB_EDTYPE, "dtype %d is neither HYB_F32 nor HYB_BF16", d->dtype);
  if (d->tokens < 0 || d->batch < 0) return fail(HYB_EINVAL, "tokens %d and batch %d must be >= 0", d->tokens, d->batch);
  if (d->n_kv_heads < 1 || d->n_kv_heads > 65536)
    return fail(HYB_EINVAL, "n_kv_heads %d is not in 1 .. 65536", d->n_kv_heads);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(HYB_EUNSUPPORTED, "head_dim %d not supported (64 or 128)", d->head_dim);
  hyb::KvQ8Args a{};
  TRY(check_page(d->page_size, d->scale_block, d->max_pages, d->n_pages, &a.page_shift, &a.sb_shift));
  const long n = (long)d->n_kv_heads * d->head_dim;
  for (const int64_t s : {d->k_stride, d->v_stride}) {
    if (s != 0 && (s < n || s > (1L << 31)))
      return fail(HYB_EINVAL, "a row stride of %ld is shorter than the row, or longer than 2^31", (long)s);
    if (s % 8) return fail(HYB_EALIGN, "a row stride of %ld is not a multiple of 8 elements", (long)s);
  }
  a.k_stride = d->k_stride ? d->k_stride : n;
  a.v_stride = d->v_stride ? d->v_stride : n;
  a.N = d->tokens, a.B = d->batch, a.Hkv = d->n_kv_heads, a.D = d->head_dim, a.dtype = d->dtype;
  a.max_pages = d->max_pages, a.n_pages = d->n_pages;
  if (hyb::kv_q8_threads(a) > 0xffffffffL) return fail(HYB_EINVAL, "tokens * heads exceeds the grid limit");
  if (a.N == 0 || a.B == 0 || a.max_pages == 0) return ok();
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(k_pages, "k_pages"));
  TRY(check_ptr(v_pages, "v_pages"));
  TRY(check_ptr(k_scales, "k_scales"));
  TRY(check_ptr(v_scales, "v_scales"));
  TRY(check_ptr(page_table, "page_table"));
  TRY(check_ptr(first, "first"));
  TRY(check_ptr(token_start, "token_start"));
  const size_t es = elem_bytes(a.dtype), rows = (size_t)a.n_pages << a.page_shift;
  const size_t nc = rows * n, ns = (rows >> a.sb_shift) * a.Hkv;
  const Rows tok[2] = {{k, n * es, a.k_stride * es}, {v, n * es, a.v_stride * es}};
  const Buf pools[4] = {{k_pages, nc}, {v_pages, nc}, {k_scales, ns}, {v_scales, ns}};
  const Buf small[3] = {{page_table, (size_t)a.B * a.max_pages * 4}, {first, (size_t)a.B * 4},
                        {token_start, ((size_t)a.B + 1) * 4}};
  if (read) {
    TRY(check_rows(tok, 2, nullptr, 0, a.N));
    TRY(check_buffers(pools, 4, false, tok, 2, a.N));
    TRY(check_buffers(small, 3, false, tok, 2, a.N));
  } else {
    TRY(check_buffers(pools, 4, true, tok, 2, a.N));
    TRY(check_overlaps(pools, 4, small, 3));
  }
  a.k = const_cast<void*>(k), a.v = const_cast<void*>(v);  // (read by the write)
  a.page_table = page_table, a.first = first, a.token_start = token_start;
  a.k_pages = (uint8_t*)const_cast<void*>(k_pages), a.v_pages = (uint8_t*)const_cast<void*>(v_pages);
  a.k_scales = const_cast<uint8_t*>(k_scales), a.v_scales = const_cast<uint8_t*>(v_scales);
  (void)hipGetLastError();
  return launched(read ? hyb::launch_kv_q8_read(a, (hipStream_t)stream) : hyb::launch_kv_q8_write(a, (hipStream_t)stream),
                  name);
}

}  // namespace

extern "C" {

int kv_pages_q8_write(const hyb_kv_q8_dims_t* dims, const void* k, const void* v, void* k_pages, void* v_pages,
                      uint8_t* k_scales, uint8_t* v_scales, const int32_t* page_table, const int32_t* first,
                      const int32_t* token_start, void* stream) {
  return kv_q8_impl(dims, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first, token_start, false, stream);
}

int kv_pages_q8_read(const hyb_kv_q8_dims_t* dims, const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                     const uint8_t* v_scales, const int32_t* page_table, const int32_t* first,
                     const int32_t* token_start, void* k, void* v, void* stream) {
  return kv_q8_impl(dims, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first, token_start, true, stream);
}

int softmax_window_step_paged_q8(const hyb_dims_t* dims, const void* q, const void* k, const void* v,
                                 const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                                 const uint8_t* v_scales, int32_t n_pages, int32_t page_size, int32_t scale_block,
                                 const int32_t* page_table, int32_t max_pages, const int32_t* prefix_len,
                                 int32_t window, int32_t n_sinks, const int32_t* block_len, void* out, void* ws,
                                 size_t ws_bytes, void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, false, &s));
  TRY(no_step_flags(dims));
  if (window < 0 || n_sinks < 0)
    return fail(HYB_EINVAL, "window %d and n_sinks %d must be >= 0", window, n_sinks);
  if (s.Hq > 65536) return fail(HYB_EUNSUPPORTED, "n_q_heads %d not supported (at most 65536)", s.Hq);
  int page_shift, sb_shift;
  TRY(check_page(page_size, scale_block, max_pages, n_pages, &page_shift, &sb_shift));
  if (s.B == 0) return ok();
  const int max_prefix = max_pages * page_size;
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(prefix_len, "prefix_len"));
  TRY(check_ptr(k_pages, "k_pages", max_prefix > 0));
  TRY(check_ptr(v_pages, "v_pages", max_prefix > 0));
  TRY(check_ptr(k_scales, "k_scales", max_prefix > 0));
  TRY(check_ptr(v_scales, "v_scales", max_prefix > 0));
  TRY(check_ptr(page_table, "page_table", max_prefix > 0));
  TRY(check_ptr(block_len, "block_len", false));
  // cached tokens that a query sees, at most (a window's ends share tiles with hidden tokens)
  const int max_seen = (int)std::min<long long>(max_prefix, (long long)window + n_sinks + 64);
  const size_t need = hybrid_workspace_bytes(dims, HYB_OP_WINDOW_STEP_Q8, max_seen);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(HYB_EWORKSPACE, "softmax_window_step_paged_q8 needs %zu workspace bytes, got %zu", need,
                ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws", false));
  const hyb::SoftmaxQ8Args a{{s, q, k, v, k_pages, v_pages, prefix_len, max_prefix, out, ws,
                              hyb::softmax_q8_splits(s, max_seen + 32), page_table, page_shift, max_pages, n_pages,
                              max_seen + 32, window, n_sinks, block_len},
                             k_scales, v_scales, sb_shift};
  if (hyb::softmax_q8_threads(a) > 0xffffffffL)
    return fail(HYB_EINVAL, "batch * heads * block exceeds the grid limit");
  const size_t es = elem_bytes(s.dtype), nq = (size_t)s.B * s.L * s.Hq * s.D, nkv = (size_t)s.B * s.L * s.Hkv * s.D;
  const size_t rows = max_prefix > 0 ? (size_t)n_pages << page_shift : 0;
  const size_t nc = rows * s.Hkv * s.D, ns = (rows >> sb_shift) * s.Hkv;
  const Buf written[] = {{out, nq * out_bytes(s)}, {ws, need}};
  const Buf read_only[] = {{q, nq * es}, {k, nkv * es}, {v, nkv * es}, {k_pages, nc}, {v_pages, nc}, {k_scales, ns},
                           {v_scales, ns}, {page_table, (size_t)s.B * max_pages * 4}, {prefix_len, (size_t)s.B * 4},
                           {block_len, (size_t)s.B * 4}};
  TRY(check_overlaps(written, 2, read_only, 10));
  (void)hipGetLastError();
  return launched(hyb::launch_softmax_q8(a, (hipStream_t)stream), "softmax_window_step_paged_q8");
}

}  // extern "C"

namespace {

// What softmax_packed_prefill and its gradient check alike.
int check_packed(const hyb_dims_t* dims, int32_t tokens, int32_t window, int32_t n_sinks, int64_t q_stride,
                 int64_t k_stride, int64_t v_stride, hyb::PackedArgs* a) {
  hyb::Shape& s = a->s;
  TRY(check_dims(dims, false, &s));
  TRY(no_step_flags(dims));
  if (tokens < 0 || tokens > (1 << 30)) return fail(HYB_EINVAL, "tokens %d is not in 0 .. 2^30", tokens);
  if (window < 0 || n_sinks < 0)
    return fail(HYB_EINVAL, "window %d and n_sinks %d must be >= 0", window, n_sinks);
  if (s.Hq > 65536) return fail(HYB_EUNSUPPORTED, "n_q_heads %d not supported (at most 65536)", s.Hq);
  const long nq = (long)s.Hq * s.D, nk = (long)s.Hkv * s.D;
  const int64_t given[3] = {q_stride, k_stride, v_stride};
  const long least[3] = {nq, nk, nk};
  long* set[3] = {&a->q_stride, &a->k_stride, &a->v_stride};
  for (int i = 0; i < 3; ++i) {
    // (a tile of 32 rows is addressed with 32 bits)
    if (given[i] != 0 && (given[i] < least[i] || given[i] > (1L << 24)))
      return fail(HYB_EINVAL, "a row stride of %ld is shorter than the row, or longer than 2^24", (long)given[i]);
    if (given[i] % 8) return fail(HYB_EALIGN, "a row stride of %ld is not a multiple of 8 elements", (long)given[i]);
    *set[i] = given[i] ? given[i] : least[i];
  }
  if (s.B > 0 && tokens > 0 && hyb::packed_threads(s, tokens) > 0xffffffffL)
    return fail(HYB_EINVAL, "tokens * heads exceeds the grid limit");
  a->N = tokens, a->window = window, a->n_sinks = n_sinks;
  return HYB_OK;
}

}  // namespace

extern "C" {

int softmax_packed_prefill(const hyb_dims_t* dims, int32_t tokens, int32_t window, int32_t n_sinks, const void* q,
                           const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                           const int32_t* token_start, void* out, float* lse, void* stream) {
  hyb::PackedArgs a{};
  TRY(check_packed(dims, tokens, window, n_sinks, q_stride, k_stride, v_stride, &a));
  const hyb::Shape& s = a.s;
  if (s.B == 0 || tokens == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(token_start, "token_start"));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(lse, "lse", false));
  const size_t es = elem_bytes(s.dtype), n = tokens;
  const size_t nq = (size_t)s.Hq * s.D, nk = (size_t)s.Hkv * s.D;
  const Rows in[3] = {{q, nq * es, a.q_stride * es}, {k, nk * es, a.k_stride * es}, {v, nk * es, a.v_stride * es}};
  const Buf written[2] = {{out, n * nq * out_bytes(s)}, {lse, n * s.Hq * 4}};
  const Buf small[1] = {{token_start, ((size_t)s.B + 1) * 4}};
  TRY(check_buffers(written, 2, true, in, 3, tokens));
  TRY(check_overlaps(written, 2, small, 1));
  a.q = q, a.k = k, a.v = v, a.token_start = token_start;
  a.out = out, a.lse = lse;
  (void)hipGetLastError();
  return launched(hyb::launch_packed_prefill(a, (hipStream_t)stream), "softmax_packed_prefill");
}

int softmax_packed_backward(const hyb_dims_t* dims, int32_t tokens, int32_t window, int32_t n_sinks, const void* q,
                            const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                            const int32_t* token_start, const void* out, const float* lse, const void* dout, void* dq,
                            void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
  hyb::PackedArgs a{};
  TRY(check_packed(dims, tokens, window, n_sinks, q_stride, k_stride, v_stride, &a));
  const hyb::Shape& s = a.s;
  if (s.B == 0 || tokens == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(token_start, "token_start"));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(lse, "lse"));
  TRY(check_ptr(dout, "dout"));
  TRY(check_ptr(dq, "dq"));
  TRY(check_ptr(dk, "dk"));
  TRY(check_ptr(dv, "dv"));
  const size_t need = hybrid_workspace_bytes(dims, HYB_OP_PACKED_BACKWARD, tokens);
  if (!ws || ws_bytes < need)
    return fail(HYB_EWORKSPACE, "softmax_packed_backward needs %zu workspace bytes, got %zu", need,
                ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws"));
  const size_t es = elem_bytes(s.dtype), eo = out_bytes(s), n = tokens;
  const size_t nq = (size_t)s.Hq * s.D, nk = (size_t)s.Hkv * s.D;
  const Rows in[3] = {{q, nq * es, a.q_stride * es}, {k, nk * es, a.k_stride * es}, {v, nk * es, a.v_stride * es}};
  const Buf written[4] = {{dq, n * nq * eo}, {dk, n * nk * eo}, {dv, n * nk * eo}, {ws, need}};
  const Buf read_only[4] = {{out, n * nq * es}, {dout, n * nq * es}, {lse, n * s.Hq * 4},
                            {token_start, ((size_t)s.B + 1) * 4}};
  TRY(check_buffers(written, 4, true, in, 3, tokens));
  TRY(check_overlaps(written, 4, read_only, 4));
  a.q = q, a.k = k, a.v = v, a.token_start = token_start;
  a.out = const_cast<void*>(out), a.lse = const_cast<float*>(lse);  // (only read)
  a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv, a.ws = (float*)ws;
  (void)hipGetLastError();
  return launched(hyb::launch_packed_backward(a, (hipStream_t)stream), "softmax_packed_backward");
}

}  // extern "C"

namespace {

// Validation and dispatch of the backward; dq, dk, dv all null (the Stage-1
// gradient only) or all set (the input gradients as well).
int backward_impl(const hyb_dims_t* dims, int32_t seq_len, const void* q,
                  const void* k, const void* v, const void* W,
                  const float* alpha, const void* dout, const void* target,
                  float* dq, float* dk, float* dv, bool inputs, float* dW,
                  float* dalpha, float* loss, void* ws, size_t ws_bytes,
                  void* stream) {
  hyb::Shape s;
  TRY(check_dims(dims, false, &s));
  if (dims->flags != 0) return fail(HYB_EINVAL, "flags must be 0 for the backward");
  if (!hyb::backward_supported(s))
    return fail(HYB_EUNSUPPORTED, "backward supports feat_dim 64 or 128, not %d",
                2 * s.F);
  if (seq_len <= 0 || seq_len % s.L != 0)
    return fail(HYB_EINVAL, "seq_len %d is not a positive multiple of block %d",
                seq_len, s.L);
  if (s.B == 0) return ok();
  TRY(check_ptr(q, "q"));
  TRY(check_ptr(k, "k"));
  TRY(check_ptr(v, "v"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(alpha, "alpha"));
  TRY(check_ptr(dout, "dout", false));
  TRY(check_ptr(target, "target", false));
  if ((dout == nullptr) == (target == nullptr))
    return fail(HYB_EINVAL, "exactly one of dout and target must be given");
  if (dout && loss) return fail(HYB_EINVAL, "loss needs a target");
  if (inputs) {
    TRY(check_ptr(dq, "dq"));
    TRY(check_ptr(dk, "dk"));
    TRY(check_ptr(dv, "dv"));
  }
  TRY(check_ptr(dW, "dW"));
  TRY(check_ptr(dalpha, "dalpha"));
  TRY(check_ptr(loss, "loss", false));
  const size_t need = hybrid_workspace_bytes(
      dims, inputs ? HYB_OP_BACKWARD_FULL : HYB_OP_BACKWARD, seq_len);
  if (!ws || ws_bytes < need)
    return fail(HYB_EWORKSPACE, "backward needs %zu workspace bytes, got %zu",
                need, ws ? ws_bytes : (size_t)0);
  TRY(check_ptr(ws, "ws"));
  const size_t es = elem_bytes(s.dtype);
  const size_t nq = (size_t)s.B * seq_len * s.Hq * s.D * es;
  const size_t nkv = (size_t)s.B * seq_len * s.Hkv * s.D * es;
  const size_t nW = (size_t)s.Hq * s.F * s.D * es;
  const size_t nq4 = (size_t)s.B * seq_len * s.Hq * s.D * 4;
  const size_t nkv4 = (size_t)s.B * seq_len * s.Hkv * s.D * 4;
  struct Buf {
    const void* p;
    size_t n;
  };
  const Buf written[7] = {{dW, (size_t)s.Hq * s.F * s.D * 4},
                          {dalpha, (size_t)s.Hq * 4},
                          {loss, (size_t)s.Hq * 4},
                          {ws, need},
                          {dq, nq4},
                          {dk, nkv4},
                          {dv, nkv4}};
  const Buf read_only[6] = {{q, nq},  {k, nkv}, {v, nkv}, {W, nW},
                            {alpha, (size_t)s.Hq * 4},
                            {dout ? dout : target, nq}};
  for (int i = 0; i < 7; ++i) {
    for (int j = i + 1; j < 7; ++j)
      if (overlap(written[i].p, written[i].n, written[j].p, written[j].n))
        return fail(HYB_EINVAL, "outputs or the workspace overlap each other");
    for (int j = 0; j < 6; ++j)
      if (overlap(written[i].p, written[i].n, read_only[j].p, read_only[j].n))
        return fail(HYB_EINVAL, "an output or the workspace overlaps an input");
  }
  hyb::BackwardArgs a{s, seq_len, q, k, v, W, alpha, dout, target,
                      dW, dalpha, loss, ws};
  if (inputs) {
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
  }
  (void)hipGetLastError();
  return launched(hyb::launch_backward(a, (hipStream_t)stream), "backward");
}

}  // namespace

extern "C" {

int hybrid_attn_backward(const hyb_dims_t* dims, int32_t seq_len,
                         const void* q, const void* k, const void* v,
                         const void* W, const float* alpha, const void* dout,
                         const void* target, float* dW, float* dalpha,
                         float* loss, void* ws, size_t ws_bytes, void* stream) {
  return backward_impl(dims, seq_len, q, k, v, W, alpha, dout, target, nullptr,
                       nullptr, nullptr, false, dW, dalpha, loss, ws, ws_bytes,
                       stream);
}

int hybrid_attn_backward_full(const hyb_dims_t* dims, int32_t seq_len,
                              const void* q, const void* k, const void* v,
                              const void* W, const float* alpha,
                              const void* dout, const void* target, float* dq,
                              float* dk, float* dv, float* dW, float* dalpha,
                              float* loss, void* ws, size_t ws_bytes,
                              void* stream) {
  return backward_impl(dims, seq_len, q, k, v, W, alpha, dout, target, dq, dk,
                       dv, true, dW, dalpha, loss, ws, ws_bytes, stream);
}

size_t hybrid_workspace_bytes(const hyb_dims_t* dims, int32_t op,
                              int32_t extent) {
  hyb::Shape s;
  const std::string saved = g_err;
  const int rc = check_dims(dims, false, &s);
  g_err = saved;
  if (rc != HYB_OK || extent < 0) return 0;
  switch (op) {
    case HYB_OP_STEP:
    case HYB_OP_COMMIT:
      return 0;
    case HYB_OP_PREFILL:
      if (extent == 0 || extent % s.L != 0) return 0;
      return hyb::prefill_ws_bytes(s, extent);
    case HYB_OP_WINDOW_STEP:
      return hyb::softmax_prefix_ws_bytes(s, hyb::softmax_window_splits(s, extent));
    case HYB_OP_PACKED_BACKWARD:
      return s.B > 0 && extent > 0 && extent <= (1 << 30) ? hyb::packed_backward_ws_bytes(s, extent) : 0;
    case HYB_OP_WINDOW_STEP_Q8:
      if (extent > 0x7fffffff - 64) return 0;
      return hyb::softmax_prefix_ws_bytes(s, hyb::softmax_q8_splits(s, extent + 32));
    case HYB_OP_SOFTMAX_PREFIX:
      return hyb::softmax_prefix_ws_bytes(
          s, hyb::softmax_prefix_splits(s, extent));
    case HYB_OP_BACKWARD:
    case HYB_OP_BACKWARD_FULL:
      if (extent == 0 || extent % s.L != 0 || !hyb::backward_supported(s)) return 0;
      return hyb::backward_ws_bytes(s, extent, op == HYB_OP_BACKWARD_FULL);
    case HYB_OP_WINDOW_PREFILL:
      return 0;
    case HYB_OP_WINDOW_BACKWARD:
      return s.B > 0 && extent > 0 && extent <= (1 << 30) ? hyb::window_backward_ws_bytes(s, extent) : 0;
  }
  return 0;
}

const char* hybrid_last_error(void) { return g_err.c_str(); }

}  // extern "C"
