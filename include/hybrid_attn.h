/*
 * hybrid_attn.h -- C ABI of libhybattn, the MI355X (gfx950) block-hybrid
 * attention library.
 *
 * Method: "Retrofitting Linear Attention into Diffusion Language Models",
 * Section 3.1.  For a query q of the active block, with a per-query-head
 * feature map phi(x) = [softmax(xW), softmax(-xW)] (W in R^{d x F}, so phi has
 * f = 2F entries) and a committed-context state S (f x d), Z (f):
 *   sm_num  = sum_j exp(q.k_j/sqrt(d)) v_j,   sm_den = sum_j exp(q.k_j/sqrt(d))
 *             (j over all L tokens of the active block, no mask)
 *   lin_num = phi(q)^T S,                     lin_den = phi(q)^T Z
 *   out     = (w sm_num + lin_num) / (w sm_den + lin_den),  w = sigmoid(alpha)
 * and committing a block adds sum_t phi(k_t) v_t^T to S and sum_t phi(k_t)
 * to Z.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Memory.  Every pointer argument is a device pointer (hipMalloc'ed or
 *   equivalent), owned by the caller.  The library never allocates or frees
 *   device memory; a scratch buffer, where one is needed, is the caller's
 *   workspace of at least hybrid_workspace_bytes() bytes.
 * Alignment.  Every pointer must be 16-byte aligned.
 * Layouts.  Row-major, contiguous, outermost index first:
 *   q, out        [B][L][Hq][d]        (prefill: [B][T][Hq][d])
 *   k, v          [B][L][Hkv][d]       (prefill: [B][T][Hkv][d])
 *   W             [Hq][F][d]           row j of head h is column j of W_h;
 *                                      this is the weight layout of a linear
 *                                      layer d -> F
 *   alpha         [Hq] float           gate logits; the library forms sigmoid
 *   S             [n_slots][Hq][d][f] float   S_h stored transposed:
 *                                      entry (feature r, value dim c) of S_h
 *                                      is at c*f + r, so the f features of
 *                                      one value dim are contiguous
 *   z             [n_slots][Hq][f] float
 *   slots         [B] int32 or NULL    state slot of request b; NULL means
 *                                      slot b.  A slot outside [0, n_slots)
 *                                      makes that request's outputs NaN and
 *                                      leaves every state untouched.
 *   block_len     [B] int32 or NULL    active tokens of request b's block,
 *                                      clamped to [0, L]; NULL means L for
 *                                      every request.  Request b then acts
 *                                      as a call with L = block_len[b] on
 *                                      its first block_len[b] rows: its
 *                                      later rows of q, k and v play no part
 *                                      (their values may be anything, NaN
 *                                      included) and its later rows of out
 *                                      are not written.  0 makes the request
 *                                      a no-op.  This serves a batch whose
 *                                      requests sit in blocks of different
 *                                      lengths, e.g. a prompt's last,
 *                                      partial block.
 *   k_cache, v_cache [B][max_prefix][Hkv][d]; request b uses rows
 *                                      0 .. prefix_len[b]-1.
 *   Query head h reads KV head h / (Hq / Hkv).
 * Types.  q, k, v, W and the KV cache share dims->dtype (fp32 or bf16), and so
 *   does out unless dims->flags has HYB_OUT_F32; alpha, S and z are always
 *   fp32.  All accumulation is fp32.  On the bf16 path the matrix-core
 *   operands are bf16: phi(q) and the state read by a step are rounded to
 *   bf16 (round to nearest even), while the block softmax weights and phi(k)
 *   in a state update are carried as a bf16 pair hi + lo (about 16 bits).
 *   A bf16 out is the rounded fp32 result.
 * Execution.  Work is enqueued on `stream` (a hipStream_t; NULL = the null
 *   stream) and the call returns without synchronising.  Results are
 *   bitwise reproducible from run to run (no atomics).
 * Validation.  Every check below runs on the host before anything is
 *   enqueued.  On failure the call returns the status, enqueues nothing,
 *   touches no output and sets a message readable with hybrid_last_error().
 *   Values that live in device memory (slots, block_len, prefix_len) cannot be checked
 *   on the host; the kernels clamp or mask them as documented per call.
 * Errors after launch.  HYB_ELAUNCH reports a failed kernel launch; outputs,
 *   and for commit/prefill the state, are then undefined.
 * Threading.  Calls are reentrant; the error message is thread-local.
 */
#ifndef HYBRID_ATTN_H
#define HYBRID_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HYB_OK = 0,
  HYB_ENULL = 1,        /* a required pointer is NULL                       */
  HYB_EINVAL = 2,       /* a size is out of range or inconsistent           */
  HYB_EALIGN = 3,       /* a pointer is not 16-byte aligned                 */
  HYB_EDTYPE = 4,       /* dims->dtype is not a hyb_dtype_t                 */
  HYB_EUNSUPPORTED = 5, /* no kernel for this (dtype, head_dim, feat_dim)   */
  HYB_EWORKSPACE = 6,   /* workspace missing or smaller than required       */
  HYB_ELAUNCH = 7       /* the HIP runtime rejected a launch                */
} hyb_status_t;

typedef enum { HYB_F32 = 0, HYB_BF16 = 1 } hyb_dtype_t;

typedef enum {
  HYB_OP_STEP = 0,
  HYB_OP_COMMIT = 1,
  HYB_OP_PREFILL = 2,
  HYB_OP_SOFTMAX_PREFIX = 3,
  HYB_OP_BACKWARD = 4,
  HYB_OP_BACKWARD_FULL = 5,
  HYB_OP_WINDOW_STEP = 6,
  HYB_OP_WINDOW_PREFILL = 7,
  HYB_OP_WINDOW_BACKWARD = 8,
  HYB_OP_WINDOW_STEP_Q8 = 9,
  HYB_OP_PACKED_BACKWARD = 10
} hyb_op_t;

typedef struct {
  int32_t batch;      /* B, requests in this call, >= 0 (0: nothing to do)   */
  int32_t n_q_heads;  /* Hq, >= 1                                            */
  int32_t n_kv_heads; /* Hkv, >= 1, divides Hq                               */
  int32_t head_dim;   /* d: 64 or 128                                        */
  int32_t block;      /* L, active-block tokens: 1..32                       */
  int32_t feat_dim;   /* f = 2F, rows of S: 64, 128 or 256                   */
  int32_t dtype;      /* hyb_dtype_t                                         */
  int32_t n_slots;    /* rows of the state pool S, z; >= 1 when batch > 0   */
  int32_t flags;      /* HYB_OUT_F32 and, for the step only, HYB_STEP_SPLIT
                         or HYB_STEP_WHOLE; any other bit is rejected      */
} hyb_dims_t;

/* flags: out is fp32 whatever dtype is (default: out has dtype).  The bf16
 * output of a call equals the round-to-nearest-even bf16 of its fp32 output
 * bit for bit. */
#define HYB_OUT_F32 1
/* flags of hybrid_attn_step only (any other entry point rejects them): which
 * of its three kernels runs.  HYB_STEP_SPLIT: one wave per (request, query
 * head, 32-column slice of d), for batches too small to fill the chip with
 * HYB_STEP_WHOLE: one workgroup per group of query heads sharing a KV head,
 * each streaming its heads' whole states.  HYB_STEP_HALVES: two workgroups
 * per group of four query heads, each streaming half of every head's state
 * columns and writing half of its output columns (bf16, feat_dim <= 128,
 * n_q_heads / n_kv_heads a multiple of 4; otherwise HYB_EUNSUPPORTED).  None:
 * the library picks by the batch (HALVES where it is supported and its
 * workgroups fill 128 to 256 compute units; else SPLIT while its
 * B * Hq * d/32 waves fit on the chip at once, 1024 of them; else HALVES
 * while its workgroups fit on the 256 compute units; else WHOLE).  More than
 * one: rejected.
 * Results agree to the same bound against the definition; they need not
 * agree bit for bit. */
#define HYB_STEP_SPLIT 2
#define HYB_STEP_WHOLE 4
#define HYB_STEP_HALVES 8

/* One denoising step of the active block (Section 3.1: within-block
 * softmax branch, linear readout of the committed state, gated merge with a
 * shared normaliser).  Reads S and z, writes out.  q, k, v, W, alpha, S, z
 * and out are required; slots and block_len may be NULL.  out must not
 * overlap an input.  Empty context (z = 0) gives plain block softmax. */
int hybrid_attn_step(const hyb_dims_t* dims, const void* q, const void* k,
                     const void* v, const void* W, const float* alpha,
                     const float* S, const float* z, const int32_t* slots,
                     const int32_t* block_len, void* out, void* stream);

/* The last denoising step of a block fused with its commit, in one launch
 * (the single kernel of Section 3.3: within-block softmax, readout, gated
 * merge and the causal state update).  out is exactly what hybrid_attn_step
 * gives on the state as it was; then, as hybrid_state_commit,
 * S_h += sum_t phi_h(k_t) v_t^T and z_h += sum_t phi_h(k_t), in place.
 * Arguments as for hybrid_attn_step, with S and z writable.  out, S and z
 * must not overlap each other or any input; two requests of one call must
 * not share a slot.  A request whose slot is out of range gets NaN outputs
 * and leaves the state untouched. */
int hybrid_attn_step_commit(const hyb_dims_t* dims, const void* q,
                            const void* k, const void* v, const void* W,
                            const float* alpha, float* S, float* z,
                            const int32_t* slots, const int32_t* block_len,
                            void* out, void* stream);

/* Commit of a finished block (Section 3.1 state update):
 * S_h += sum_t phi_h(k_t) v_t^T and z_h += sum_t phi_h(k_t) over the block
 * tokens (the first block_len[b] of request b; all L when block_len is
 * NULL), in place, for every request and query head.  Two requests of one
 * call must not share a slot. */
int hybrid_state_commit(const hyb_dims_t* dims, const void* k, const void* v,
                        const void* W, float* S, float* z,
                        const int32_t* slots, const int32_t* block_len,
                        void* stream);

/* Block-causal prefill of seq_len tokens (Figure 2 pattern): the tokens are
 * cut into seq_len / L blocks; block c is answered against the state of the
 * blocks before it (as hybrid_attn_step) and then committed.  The state
 * starts from what S, z hold, so successive calls continue one prompt.
 * seq_len must be a positive multiple of L.  out may be NULL (state only; q
 * is then ignored and may be NULL).  ws/ws_bytes: workspace of at least
 * hybrid_workspace_bytes(dims, HYB_OP_PREFILL, seq_len) bytes (may be NULL
 * when that is 0); the prompt is processed in sequence segments whose state
 * increments (and the states the segments start from) pass through it, so
 * results equal the block-by-block ones up to the order of fp32 additions.  It
 * must not overlap any other argument.  Two requests of one call must not share
 * a slot. */
int hybrid_state_prefill(const hyb_dims_t* dims, int32_t seq_len,
                         const void* q, const void* k, const void* v,
                         const void* W, const float* alpha, float* S, float* z,
                         const int32_t* slots, void* out, void* ws,
                         size_t ws_bytes, void* stream);

/* Bytes of the library-held scratch buffer of hybrid_state_prefill_noalloc,
 * per GPU. */
#define HYB_NOALLOC_SCRATCH_BYTES (64u << 20)

/* hybrid_state_prefill for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same computation and results, bit for bit, with the
 * workspace taken from a scratch buffer the library holds on each GPU
 * (HYB_NOALLOC_SCRATCH_BYTES, kept from the first call on a device until
 * the process ends).  The call itself allocates nothing; the caller still
 * passes inputs, outputs and the state.  A call whose workspace
 * (hybrid_workspace_bytes(dims, HYB_OP_PREFILL, seq_len)) exceeds the
 * scratch size returns HYB_EWORKSPACE and enqueues nothing.  Every call on
 * one GPU shares that GPU's buffer, which keeps the last call's contents
 * (nothing in it needs to start at zero): calls whose executions overlap on
 * one GPU, e.g. on two streams, race and must not be issued. */
int hybrid_state_prefill_noalloc(const hyb_dims_t* dims, int32_t seq_len,
                                 const void* q, const void* k, const void* v,
                                 const void* W, const float* alpha, float* S,
                                 float* z, const int32_t* slots, void* out,
                                 void* stream);

/* Exact softmax attention of the active block's queries over each request's
 * cached prefix plus the block itself (the softmax teacher the hybrid layer
 * replaces; Section 2.2, without a mask inside the block).  prefix_len is a
 * device array [B]; values are clamped to [0, max_prefix].  ws/ws_bytes: at
 * least hybrid_workspace_bytes(dims, HYB_OP_SOFTMAX_PREFIX, max_prefix)
 * bytes, not overlapping any argument; when that is 0 (the prefix is not
 * split across workgroups) ws may be NULL.  How a request's keys are split
 * follows from the lengths of all requests of the call, so the same request
 * beside others may round differently (bf16: its weights, to 2^-8 each). */
int softmax_prefix_step(const hyb_dims_t* dims, const void* q, const void* k,
                        const void* v, const void* k_cache,
                        const void* v_cache, const int32_t* prefix_len,
                        int32_t max_prefix, void* out, void* ws,
                        size_t ws_bytes, void* stream);

/* softmax_prefix_step over a paged KV cache, as a serving engine keeps it
 * (Section 3.3 keeps the hybrid state beside such a cache; the softmax
 * layers it replaces read it).  k_pages, v_pages: page pools
 * [n_pages][page_size][Hkv][d] in dims->dtype; page_table: device
 * [B][max_pages] int32, entry i of request b naming the page that holds its
 * cached tokens i*page_size .. (i+1)*page_size - 1 (token j at row
 * j % page_size).  prefix_len (device [B]) is clamped to
 * [0, max_pages * page_size]; only the first ceil(prefix_len[b] / page_size)
 * entries of a row are read, and a page number outside [0, n_pages) is
 * clamped into it (device values cannot be checked on the host).  page_size
 * is a power of two from 32 to 65536 (HYB_EUNSUPPORTED otherwise); n_pages
 * >= 1 and the page table are required when max_pages > 0.  Pages may be
 * shared by requests and appear in any order.  The result equals
 * softmax_prefix_step on the gathered contiguous cache, bit for bit.
 * ws/ws_bytes: at least hybrid_workspace_bytes(dims, HYB_OP_SOFTMAX_PREFIX,
 * max_pages * page_size) bytes (NULL when that is 0), not overlapping any
 * argument.  out must not overlap an input. */
int softmax_prefix_step_paged(const hyb_dims_t* dims, const void* q,
                              const void* k, const void* v,
                              const void* k_pages, const void* v_pages,
                              int32_t n_pages, int32_t page_size,
                              const int32_t* page_table, int32_t max_pages,
                              const int32_t* prefix_len, void* out, void* ws,
                              size_t ws_bytes, void* stream);

/* Gradient of the block-hybrid layer over a training sequence with respect
 * to its feature-map weights W and gate logits alpha: the attention transfer
 * of Section 3.2 (Stage 1), which trains only {W, alpha} with the backbone
 * frozen.  The forward is the block-causal pattern of Figure 2 from an empty
 * state (hybrid_state_prefill's outputs for a fresh request): q [B][T][Hq][d],
 * k, v [B][T][Hkv][d], W, alpha as for hybrid_attn_step, T = seq_len.
 * Objective, exactly one of:
 *   dout   [B][T][Hq][d] (dims->dtype): L = sum <dout, out>, i.e. the
 *          gradient for an upstream gradient dout; loss must be NULL;
 *   target [B][T][Hq][d] (dims->dtype): the frozen softmax teacher's output;
 *          L = sum |out - target|^2, the attention-transfer loss, formed
 *          without writing out; loss (fp32 [Hq], may be NULL) receives L per
 *          query head.
 * Outputs (fp32, overwritten, summed over the batch): dW [Hq][F][d] in W's
 * layout, dalpha [Hq].  seq_len must be a positive multiple of L.  feat_dim
 * must be 64 or 128 (HYB_EUNSUPPORTED otherwise); dims->flags must be 0;
 * n_slots is not used.  ws/ws_bytes: at least hybrid_workspace_bytes(dims,
 * HYB_OP_BACKWARD, seq_len) bytes, not overlapping any argument; outputs
 * must not overlap each other or an input.  batch 0 writes nothing.
 * Deterministic: partial sums are added in a fixed order. */
int hybrid_attn_backward(const hyb_dims_t* dims, int32_t seq_len,
                         const void* q, const void* k, const void* v,
                         const void* W, const float* alpha, const void* dout,
                         const void* target, float* dW, float* dalpha,
                         float* loss, void* ws, size_t ws_bytes, void* stream);

/* hybrid_attn_backward that also returns the gradients with respect to the
 * layer's inputs q, k and v, which end-to-end training through the hybrid
 * layers needs (Stage 2 of Section 3.2 adapts the attention projections
 * around them).  Arguments and the objective as for hybrid_attn_backward;
 * dq [B][T][Hq][d], dk and dv [B][T][Hkv][d] are fp32 whatever dims->dtype
 * is (dk and dv sum over the query heads that share each KV head), all
 * three required and overwritten.  ws/ws_bytes: at least
 * hybrid_workspace_bytes(dims, HYB_OP_BACKWARD_FULL, seq_len) bytes.  No
 * output may overlap another output, an input or the workspace.  The
 * in-block softmax weights are formed as exp(log w + q.k/sqrt(d)), so the
 * scaled scores must stay well below 80 (the W, alpha gradients share this
 * range through 1/D).  Deterministic. */
int hybrid_attn_backward_full(const hyb_dims_t* dims, int32_t seq_len,
                              const void* q, const void* k, const void* v,
                              const void* W, const float* alpha,
                              const void* dout, const void* target, float* dq,
                              float* dk, float* dv, float* dW, float* dalpha,
                              float* loss, void* ws, size_t ws_bytes,
                              void* stream);

/* softmax_prefix_step_paged for a layer that attends to a window of the cache
 * and its first tokens: of request b's cached tokens the active block's queries
 * see the last `window` and the first n_sinks (all of them where those
 * overlap), and the whole block.  A cached token's distance counts from the
 * block's start, so every query of the block sees the same ones; a block of one
 * token (L = 1) is autoregressive decoding with a window of window + 1 tokens.
 * window and n_sinks are >= 0; a window of at least the prefix gives
 * softmax_prefix_step_paged.  block_len (device [B] or NULL): active tokens of
 * each block, as for hybrid_attn_step.
 * Arguments otherwise as for softmax_prefix_step_paged, rows past block_len[b]
 * are not written, and scores q.k must be below 1e29 in magnitude.  Tokens that are not
 * seen play no part, whatever their rows hold (NaN included), and of a page
 * table row only entries 0 .. ceil(min(n_sinks, prefix) / page_size) - 1 and
 * (prefix - window) / page_size (rounded down) .. ceil(prefix / page_size) - 1
 * are read, so pages that left the window may be freed and reused.
 * Up to 65536 query heads.  ws/ws_bytes: at least hybrid_workspace_bytes(dims,
 * HYB_OP_WINDOW_STEP, min(max_pages * page_size, n_sinks + window + 64)) bytes.
 * Calls whose executions may overlap (two streams, two captured graphs) need
 * workspaces of their own, here and below. */
int softmax_window_step_paged(const hyb_dims_t* dims, const void* q,
                              const void* k, const void* v,
                              const void* k_pages, const void* v_pages,
                              int32_t n_pages, int32_t page_size,
                              const int32_t* page_table, int32_t max_pages,
                              const int32_t* prefix_len, int32_t window,
                              int32_t n_sinks, const int32_t* block_len,
                              void* out, void* ws, size_t ws_bytes,
                              void* stream);

/* The same attention over whole sequences (block-causal, Figure 2 pattern with
 * softmax): token i of the block that starts at s = (i / L) * L sees the tokens
 * j < s + L with j >= s - window or j < n_sinks.  L = 1 is causal attention
 * with a window of window + 1 tokens; window >= seq_len is full block-causal
 * softmax, the teacher whose outputs hybrid_attn_backward takes as target.
 * q, out [B][T][Hq][d], k, v [B][T][Hkv][d], T = seq_len >= 1 (any, at most
 * 2^30; the last block may be partial).  seq_lens (device [B] or NULL): tokens
 * of each sequence, clamped to [0, T]; later rows of q, k, v play no part
 * (their values may be anything) and later rows of out and lse are not
 * written.  The values of a sequence's own tokens must be finite, also where a
 * query does not see them, and scores q.k below 1e29 in magnitude.  lse (fp32
 * [B][Hq][T], or NULL): log of the sum of exp(q.k / sqrt(d)) over the tokens
 * seen, which the gradient takes.  Up to 65536 query heads; feat_dim and n_slots
 * are not used (feat_dim must still be valid).  ws/ws_bytes: at least
 * hybrid_workspace_bytes(dims, HYB_OP_WINDOW_PREFILL, seq_len) bytes (NULL when
 * that is 0).  out and lse must not overlap each other, an input or the workspace.
 * bf16: the weights enter P V rounded to bf16, lse sums them unrounded. */
int softmax_window_prefill(const hyb_dims_t* dims, int32_t seq_len,
                           int32_t window, int32_t n_sinks, const void* q,
                           const void* k, const void* v,
                           const int32_t* seq_lens, void* out, float* lse,
                           void* ws, size_t ws_bytes, void* stream);

/* Gradient of softmax_window_prefill with respect to q, k and v for the
 * upstream gradient dout [B][T][Hq][d] (dims->dtype).  out (dims->dtype) and
 * lse are what the forward call left.  dq [B][T][Hq][d], dk, dv [B][T][Hkv][d]
 * in dims->dtype, or fp32 with HYB_OUT_F32 (on bf16 the weights and dS enter
 * the products rounded to bf16 all the same); dk and dv sum over the query
 * heads that share a KV head.  All three are required and overwritten; rows
 * past seq_lens[b] are zero.  ws/ws_bytes: at least hybrid_workspace_bytes(dims,
 * HYB_OP_WINDOW_BACKWARD, seq_len) bytes.  No output may overlap another
 * output, an input or the workspace.  Deterministic (no atomics). */
int softmax_window_backward(const hyb_dims_t* dims, int32_t seq_len,
                            int32_t window, int32_t n_sinks, const void* q,
                            const void* k, const void* v,
                            const int32_t* seq_lens, const void* out,
                            const float* lse, const void* dout, void* dq,
                            void* dk, void* dv, void* ws, size_t ws_bytes,
                            void* stream);

/* Norm and rotation of queries and keys -- what stands between the projections
 * and every attention entry point of this library. */
typedef enum {
  HYB_ROPE_HALF = 0,       /* pair i: entries i and i + rot_dim/2           */
  HYB_ROPE_INTERLEAVED = 1 /* pair i: entries 2i and 2i + 1                 */
} hyb_rope_layout_t;

typedef struct {
  int32_t tokens;     /* N >= 0 (0: nothing to do; the gradient of the
                         weights is then zero)                               */
  int32_t n_q_heads;  /* Hq >= 1                                             */
  int32_t n_kv_heads; /* Hkv >= 1                                            */
  int32_t head_dim;   /* d: 64 or 128                                        */
  int32_t rot_dim;    /* entries of a head that are rotated: its first
                         rot_dim, a multiple of 8 from 0 to d                */
  int32_t layout;     /* hyb_rope_layout_t                                   */
  int32_t dtype;      /* hyb_dtype_t of q, k, v, the weights and the pages   */
  int32_t grad_dtype; /* hyb_dtype_t of dq_out, dk_out (gradient only)       */
  int32_t flags;      /* 0 or HYB_OUT_F32: q_out, k_out, dq, dk are fp32     */
  float eps;          /* added to the mean square, > 0                       */
  float rot_scale;    /* scales sine and cosine (1 unless the position
                         scaling asks for another), finite                   */
  /* elements from a token's row to the next; 0: contiguous.  A multiple of 8,
   * at least the row's length. */
  int64_t q_stride, k_stride, v_stride; /* of the inputs                     */
  int64_t q_out_stride, k_out_stride;   /* of q_out, k_out, dq, dk           */
} hyb_rope_dims_t;

/* For every token t and head: n = x * w / sqrt(mean(x^2) + eps) over the d
 * entries, then each pair (a, b) of n's first rot_dim entries becomes
 * rot_scale * (a cos - b sin, b cos + a sin) of the angle positions[t] *
 * inv_freq[i]; the rest of n stays as it is.  q [N][Hq][d] and k [N][Hkv][d]
 * may be views of one packed projection (row strides in dims); wq, wk [d]
 * (dims->dtype), shared by the heads; NULL: that side is not normalised.
 * positions int32 [N] (any value); inv_freq double [rot_dim / 2], radians per
 * position: angles are formed in 64 bits, so far positions keep their phase, and
 * every scaling of positions for long contexts is a table (may be NULL
 * when rot_dim is 0).  Arithmetic is fp32, rounded once; a row whose sum of
 * squares leaves fp32 (about 3e38) gives zeros where it is normalised.  q_out
 * and k_out may be interleaved in one buffer, and must not overlap each other
 * or an input. */
int hybrid_qk_norm_rope(const hyb_rope_dims_t* dims, const void* q,
                        const void* k, const void* wq, const void* wk,
                        const int32_t* positions, const double* inv_freq,
                        void* q_out, void* k_out, void* stream);

/* The same with the keys and values written into a paged cache (the pools of
 * softmax_prefix_step_paged and softmax_window_step_paged): token t's k_out
 * row and its row of v [N][Hkv][d] go to row slots[t] % page_size of page slots[t] /
 * page_size, in dims->dtype.  A slot outside [0, n_pages * page_size) writes
 * nothing (tokens of a padded batch: -1).  Two tokens of one call must not
 * name the same slot.  k_out may be NULL (the block's own step needs it); other
 * rows of the pools are left as they were.  slots int32 [N] as kv_pages_plan gives them;
 * n_pages >= 1, page_size 1 or more.  The pools must not overlap each
 * other, an output or an input. */
int hybrid_qk_norm_rope_paged(const hyb_rope_dims_t* dims, const void* q,
                              const void* k, const void* v, const void* wq,
                              const void* wk, const int32_t* positions,
                              const double* inv_freq, const int32_t* slots,
                              void* q_out, void* k_out, void* k_pages,
                              void* v_pages, int32_t n_pages,
                              int32_t page_size, void* stream);

/* Gradient of hybrid_qk_norm_rope: dq, dk (with respect to q, k; rows at the
 * output strides) and dwq, dwk (fp32 [d], summed over tokens and heads,
 * overwritten; required exactly where the weight is given) for the upstream
 * gradients dq_out [N][Hq][d], dk_out [N][Hkv][d] (contiguous, grad_dtype: the
 * fp32 dq, dk of hybrid_attn_backward_full and the dq, dk of
 * softmax_window_backward fit as they are).  ws/ws_bytes: at least
 * hybrid_rope_workspace_bytes(dims) bytes when a weight is given (else may be
 * NULL).  Every token counts for dwq and dwk, so those of a padded batch need
 * finite q and k and gradients of zero.  Outputs and the workspace must not
 * overlap each other or an input.  Deterministic. */
int hybrid_qk_norm_rope_backward(const hyb_rope_dims_t* dims, const void* q,
                                 const void* k, const void* wq, const void* wk,
                                 const int32_t* positions,
                                 const double* inv_freq, const void* dq_out,
                                 const void* dk_out, void* dq, void* dk,
                                 float* dwq, float* dwk, void* ws,
                                 size_t ws_bytes, void* stream);

/* Workspace bytes of hybrid_qk_norm_rope_backward; 0 for invalid dims. */
size_t hybrid_rope_workspace_bytes(const hyb_rope_dims_t* dims);

/* Pages and cache rows of a batch's new tokens, from lengths that live on the
 * device (no host wait; a captured call plans from the lengths of each replay).
 * Request b holds prefix_len[b] cached tokens (clamped to [0, max_pages *
 * page_size]) and brings new_len[b] >= 0 more (negative: 0).  Its table row
 * page_table[b] ([B][max_pages], in and out) keeps the entries of the tokens it
 * holds; the entries its new tokens need besides take free_pages[0], [1], ..
 * in the order of the requests and of their tokens, and are written (-1 once
 * the n_free pages are used up).  Per new token, packed in the same order:
 * slots int32 [max_tokens], its row in the pools (page * page_size + row), or
 * -1 where it has no page (none left, past max_pages, or a negative or too
 * large page number in the table); positions int32 [max_tokens], its index in
 * its request.  Rows past the last token get slot -1 and position 0; tokens
 * past max_tokens are dropped (their pages are still taken).  token_start
 * int32 [B + 1]: first packed row of each request, then the total.  counts
 * int32 [2]: pages taken, pages that were missing.  Sums past 2^31 - 1 stay there,
 * and table entries past that many new pages are not written.
 * batch is 1 .. 4096 (0: nothing to do); page_size a power of two from 1 to 65536;
 * max_pages * page_size < 2^31 - 64; n_free >= 0 (free_pages may be NULL when
 * 0, and needs 4-byte alignment only: a caller goes on in its list where the
 * last call's pages ended); max_tokens >= 0 (slots and positions may be NULL
 * when 0).  Outputs must not overlap each other, the table or an input. */
int kv_pages_plan(int32_t batch, int32_t max_pages, int32_t page_size,
                  int32_t n_free, int32_t max_tokens,
                  const int32_t* prefix_len, const int32_t* new_len,
                  const int32_t* free_pages, int32_t* page_table,
                  int32_t* slots, int32_t* positions, int32_t* token_start,
                  int32_t* counts, void* stream);

/* A paged KV cache in 8 bits: half the bytes of a bf16 one, for the softmax layers
 * that keep a cache beside the hybrid ones.  k_pages, v_pages: pools of codes
 * [n_pages][page_size][Hkv][d], e4m3 (the OCP type without infinities); k_scales,
 * v_scales: [n_pages][page_size / scale_block][Hkv] bytes, the scale 2^(byte - 127)
 * of scale_block consecutive rows of a page at one KV head.  A cached value is its code
 * times its scale, also of a zeroed pool (2^-127): exactly in fp32, and in bf16 from byte 3 on
 * (below, rounded to nearest even among bf16's subnormal numbers), up to where the types
 * end.  Byte 255 is no number: the values under it are NaN, and a block that goes on keeps it.
 * page_size is a power of two from 32 to 65536, scale_block one from 32 to page_size. */
typedef struct {
  int32_t tokens;      /* N >= 0, rows of k and v (0: nothing to do)         */
  int32_t batch;       /* B >= 0, requests                                   */
  int32_t n_kv_heads;  /* Hkv, 1 .. 65536                                    */
  int32_t head_dim;    /* d: 64 or 128                                       */
  int32_t dtype;       /* hyb_dtype_t of k and v                             */
  int32_t max_pages;   /* entries of a request's page table row, >= 0        */
  int32_t n_pages;     /* pages of the pools, >= 1 when max_pages > 0        */
  int32_t page_size;   /* tokens per page                                    */
  int32_t scale_block; /* tokens per scale                                   */
  /* elements from a token's row to the next; 0: contiguous.  A multiple of 8,
   * at least the row's length. */
  int64_t k_stride, v_stride;
} hyb_kv_q8_dims_t;

/* Quantises new keys and values as it writes them into the cache.  Request b brings
 * the packed rows token_start[b] .. token_start[b + 1] - 1 of k and v [N][Hkv][d] (as
 * kv_pages_plan packs and counts them) as tokens first[b], first[b] + 1, .. of its
 * cache, through its row of page_table [B][max_pages].  Device values are clamped:
 * first [B] to [0, max_pages * page_size], token_start [B + 1] (not falling) to [0, N]
 * with token_start[0] read as 0; tokens past the page table, and those whose page
 * number lies outside [0, n_pages), are not written.
 * Per scale block and head: with m the largest finite magnitude of the block's new
 * entries, the scale is the least power of two 2^e with m <= 448 2^e, at least 2^-117;
 * where the call's first token in the block is not the block's first row, the block goes
 * on: it keeps at least its old scale, and where that grows the rows before, tokens
 * below first[b], are rounded again to the new one (exactly but for codes that become
 * subnormal).  Codes are rounded to nearest even; an entry that is not finite becomes
 * NaN.  A block's rows behind the call's last token hold nothing after a call (their
 * codes stay, their scale may not).  Requests of one call must not share a page that
 * they write to.  The pools must not overlap each other or an input. */
int kv_pages_q8_write(const hyb_kv_q8_dims_t* dims, const void* k,
                      const void* v, void* k_pages, void* v_pages,
                      uint8_t* k_scales, uint8_t* v_scales,
                      const int32_t* page_table, const int32_t* first,
                      const int32_t* token_start, void* stream);

/* The reverse: the values of cached tokens first[b], first[b] + 1, .. of request b into
 * the packed rows token_start[b] .. token_start[b + 1] - 1 of k and v, in dims->dtype.
 * Device values are clamped as above; rows of k and v without a cached token (behind the
 * last request's, past the page table, of a page number out of range) are left as they
 * were.  k and v must not overlap each other or an input (their rows may be interleaved
 * in one buffer). */
int kv_pages_q8_read(const hyb_kv_q8_dims_t* dims, const void* k_pages,
                     const void* v_pages, const uint8_t* k_scales,
                     const uint8_t* v_scales, const int32_t* page_table,
                     const int32_t* first, const int32_t* token_start, void* k,
                     void* v, void* stream);

/* softmax_window_step_paged over an 8-bit cache: q, k, v, out and the block are
 * dims->dtype, the cached tokens e4m3 with their scales.  Arguments and meaning otherwise
 * as there (a window of at least the prefix sees the whole cache), with any number of
 * query heads per KV head up to 65536 heads in all; a page number outside [0, n_pages) is
 * clamped into it.  Entries of q must be below 5e33 in magnitude (the codes' scores are summed
 * before the keys' scale is applied).  bf16: the weights enter P V rounded to bf16, their sum takes them
 * unrounded.  ws/ws_bytes: at least hybrid_workspace_bytes(dims,
 * HYB_OP_WINDOW_STEP_Q8, min(max_pages * page_size, n_sinks + window + 64)) bytes.  out and
 * the workspace must not overlap each other or an input. */
int softmax_window_step_paged_q8(
    const hyb_dims_t* dims, const void* q, const void* k, const void* v,
    const void* k_pages, const void* v_pages, const uint8_t* k_scales,
    const uint8_t* v_scales, int32_t n_pages, int32_t page_size,
    int32_t scale_block, const int32_t* page_table, int32_t max_pages,
    const int32_t* prefix_len, int32_t window, int32_t n_sinks,
    const int32_t* block_len, void* out, void* ws, size_t ws_bytes,
    void* stream);

/* softmax_window_prefill over packed sequences: dims->batch sequences of any lengths,
 * one after the other in `tokens` rows (N, 0 .. 2^30), as kv_pages_plan packs a batch's
 * prompts and a trainer its documents.  Sequence b is rows token_start[b] ..
 * token_start[b + 1] - 1 (device [B + 1], not falling; clamped to [0, N], and
 * token_start[0] read as 0); a token sees tokens of its own sequence only, as there: blocks of
 * L = dims->block count from the sequence's first token, L = 1 is causal attention, a
 * window of N or more full (block-)causal.  q [N][Hq][d], k, v [N][Hkv][d] may be views
 * of one packed projection: strides in elements from a row to the next, 0 for
 * contiguous, a multiple of 8, at most 2^24.  out [N][Hq][d] is contiguous; lse (fp32
 * [Hq][N], or NULL) as there.  Rows behind the last sequence play no part and are not
 * written.  The values of a sequence's own tokens must be finite, scores q.k below 1e29
 * in magnitude.  Up to 65536 query heads; feat_dim and n_slots are not used (feat_dim
 * must still be valid).  No workspace.  out and lse must not overlap each other or an input. */
int softmax_packed_prefill(const hyb_dims_t* dims, int32_t tokens,
                           int32_t window, int32_t n_sinks, const void* q,
                           const void* k, const void* v, int64_t q_stride,
                           int64_t k_stride, int64_t v_stride,
                           const int32_t* token_start, void* out, float* lse,
                           void* stream);

/* Gradient of softmax_packed_prefill with respect to q, k and v for the upstream
 * gradient dout [N][Hq][d] (dims->dtype); out (dims->dtype) and lse as the forward call
 * left them.  dq [N][Hq][d], dk, dv [N][Hkv][d], contiguous, in dims->dtype or fp32 with
 * HYB_OUT_F32, all required and overwritten: zero in the rows behind the last sequence
 * (a call of no sequences writes nothing).
 * ws/ws_bytes: at least hybrid_workspace_bytes(dims, HYB_OP_PACKED_BACKWARD, tokens) bytes.
 * No output may overlap another output, an input or the workspace.  Deterministic (no
 * atomics). */
int softmax_packed_backward(const hyb_dims_t* dims, int32_t tokens,
                            int32_t window, int32_t n_sinks, const void* q,
                            const void* k, const void* v, int64_t q_stride,
                            int64_t k_stride, int64_t v_stride,
                            const int32_t* token_start, const void* out,
                            const float* lse, const void* dout, void* dq,
                            void* dk, void* dv, void* ws, size_t ws_bytes,
                            void* stream);

/* Workspace bytes the given op needs for these dims; `extent` is seq_len for
 * HYB_OP_PREFILL, HYB_OP_BACKWARD, HYB_OP_BACKWARD_FULL, HYB_OP_WINDOW_PREFILL
 * and HYB_OP_WINDOW_BACKWARD, tokens for HYB_OP_PACKED_BACKWARD, max_prefix for HYB_OP_SOFTMAX_PREFIX, the cached
 * tokens a request sees at most for HYB_OP_WINDOW_STEP and
 * HYB_OP_WINDOW_STEP_Q8, ignored otherwise.
 * Returns 0 for invalid dims. */
size_t hybrid_workspace_bytes(const hyb_dims_t* dims, int32_t op,
                              int32_t extent);

/* Message of the last failed call on this thread ("" if none). */
const char* hybrid_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* HYBRID_ATTN_H */
