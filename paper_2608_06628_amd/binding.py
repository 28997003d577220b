"""ctypes binding of libhybattn (include/hybrid_attn.h), same names as the C ABI.

Argument marshalling only: shapes come from the torch tensors, pointers from
``data_ptr()``, the stream from torch's current stream, and every nonzero
status raises :class:`HybError` with the library's message.  All arithmetic
runs in the library's HIP kernels; there is no fallback path -- if the
library has not been built, loading it raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import inspect
import operator
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhybattn.so")

HYB_F32, HYB_BF16 = 0, 1
HYB_OUT_F32 = 1
HYB_STEP_SPLIT, HYB_STEP_WHOLE, HYB_STEP_HALVES = 2, 4, 8
_STEP_KERNEL = {None: 0, "auto": 0, "split": HYB_STEP_SPLIT, "whole": HYB_STEP_WHOLE,
                "halves": HYB_STEP_HALVES}
OP_STEP, OP_COMMIT, OP_PREFILL, OP_SOFTMAX_PREFIX, OP_BACKWARD, OP_BACKWARD_FULL = 0, 1, 2, 3, 4, 5
OP_WINDOW_STEP, OP_WINDOW_PREFILL, OP_WINDOW_BACKWARD = 6, 7, 8
OP_WINDOW_STEP_Q8, OP_PACKED_BACKWARD = 9, 10
_ROPE_LAYOUT = {"half": 0, "interleaved": 1}
STATUS = {0: "HYB_OK", 1: "HYB_ENULL", 2: "HYB_EINVAL", 3: "HYB_EALIGN",
          4: "HYB_EDTYPE", 5: "HYB_EUNSUPPORTED", 6: "HYB_EWORKSPACE",
          7: "HYB_ELAUNCH"}
EXPORTS = ("hybrid_attn_step", "hybrid_attn_step_commit", "hybrid_state_commit",
           "hybrid_state_prefill", "hybrid_state_prefill_noalloc", "softmax_prefix_step",
           "softmax_prefix_step_paged",
           "hybrid_attn_backward", "hybrid_attn_backward_full", "hybrid_workspace_bytes",
           "hybrid_last_error", "softmax_window_step_paged", "softmax_window_prefill",
           "softmax_window_backward", "hybrid_qk_norm_rope", "hybrid_qk_norm_rope_paged",
           "hybrid_qk_norm_rope_backward", "hybrid_rope_workspace_bytes", "kv_pages_plan",
           "kv_pages_q8_write", "kv_pages_q8_read", "softmax_window_step_paged_q8",
           "softmax_packed_prefill", "softmax_packed_backward")
NOALLOC_SCRATCH_BYTES = 64 << 20


class HybError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "block", "feat_dim",
        "dtype", "n_slots", "flags")]


class RopeDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "tokens", "n_q_heads", "n_kv_heads", "head_dim", "rot_dim", "layout", "dtype",
        "grad_dtype", "flags")] + [(n, ctypes.c_float) for n in ("eps", "rot_scale")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride",
                                      "k_out_stride")]


class KvQ8Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "tokens", "batch", "n_kv_heads", "head_dim", "dtype", "max_pages", "n_pages", "page_size",
        "scale_block")] + [(n, ctypes.c_int64) for n in ("k_stride", "v_stride")]


_lib = None


def load():
    """Load libhybattn.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with "
            "`python -m paper_2608_06628_amd.build` (no fallback exists)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    P = ctypes.POINTER(Dims)
    lib.hybrid_attn_step.argtypes = [P] + [vp] * 11
    lib.hybrid_attn_step_commit.argtypes = [P] + [vp] * 11
    lib.hybrid_state_commit.argtypes = [P] + [vp] * 8
    lib.hybrid_state_prefill.argtypes = [P, i32] + [vp] * 10 + [sz, vp]
    lib.hybrid_state_prefill_noalloc.argtypes = [P, i32] + [vp] * 10
    lib.softmax_prefix_step.argtypes = [P] + [vp] * 6 + [i32, vp, vp, sz, vp]
    lib.softmax_prefix_step_paged.argtypes = [P] + [vp] * 5 + [i32, i32, vp, i32, vp, vp, vp,
                                                                sz, vp]
    lib.hybrid_attn_backward.argtypes = [P, i32] + [vp] * 11 + [sz, vp]
    lib.hybrid_attn_backward_full.argtypes = [P, i32] + [vp] * 14 + [sz, vp]
    lib.softmax_window_step_paged.argtypes = [P] + [vp] * 5 + [i32, i32, vp, i32, vp, i32, i32,
                                                               vp, vp, vp, sz, vp]
    lib.softmax_window_prefill.argtypes = [P, i32, i32, i32] + [vp] * 7 + [sz, vp]
    lib.softmax_window_backward.argtypes = [P, i32, i32, i32] + [vp] * 11 + [sz, vp]
    R = ctypes.POINTER(RopeDims)
    lib.hybrid_qk_norm_rope.argtypes = [R] + [vp] * 9
    lib.hybrid_qk_norm_rope_paged.argtypes = [R] + [vp] * 12 + [i32, i32, vp]
    lib.hybrid_qk_norm_rope_backward.argtypes = [R] + [vp] * 13 + [sz, vp]
    lib.hybrid_rope_workspace_bytes.argtypes = [R]
    lib.hybrid_rope_workspace_bytes.restype = sz
    lib.kv_pages_plan.argtypes = [i32] * 5 + [vp] * 9
    Q = ctypes.POINTER(KvQ8Dims)
    lib.kv_pages_q8_write.argtypes = [Q] + [vp] * 10
    lib.kv_pages_q8_read.argtypes = [Q] + [vp] * 10
    lib.softmax_window_step_paged_q8.argtypes = [P] + [vp] * 7 + [i32] * 3 + [vp, i32, vp, i32, i32,
                                                                              vp, vp, vp, sz, vp]
    i64 = ctypes.c_int64
    lib.softmax_packed_prefill.argtypes = [P, i32, i32, i32, vp, vp, vp, i64, i64, i64] + [vp] * 4
    lib.softmax_packed_backward.argtypes = [P, i32, i32, i32, vp, vp, vp, i64, i64, i64] + [vp] * 8 + [sz, vp]
    lib.hybrid_workspace_bytes.argtypes = [P, i32, i32]
    lib.hybrid_workspace_bytes.restype = sz
    lib.hybrid_last_error.argtypes = []
    lib.hybrid_last_error.restype = ctypes.c_char_p
    for n in ("hybrid_attn_step", "hybrid_attn_step_commit", "hybrid_state_commit", "hybrid_state_prefill",
              "hybrid_attn_backward", "hybrid_attn_backward_full",
              "hybrid_state_prefill_noalloc", "softmax_prefix_step", "softmax_prefix_step_paged",
              "softmax_window_step_paged", "softmax_window_prefill", "softmax_window_backward",
              "hybrid_qk_norm_rope", "hybrid_qk_norm_rope_paged", "hybrid_qk_norm_rope_backward",
              "kv_pages_plan", "kv_pages_q8_write", "kv_pages_q8_read",
              "softmax_window_step_paged_q8", "softmax_packed_prefill", "softmax_packed_backward"):
        getattr(lib, n).restype = ctypes.c_int
    _lib = lib
    return lib


def last_error() -> str:
    return load().hybrid_last_error().decode()


def _check(rc: int):
    if rc != 0:
        raise HybError(rc, last_error())


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return HYB_BF16
    if t.dtype == torch.float32:
        return HYB_F32
    raise TypeError(f"unsupported activation dtype {t.dtype}")


# The host's time for a call is what a small step waits for (its kernel runs
# for about 5.5 us): the accepted tensor takes one expression, and the stream
# comes as torch's raw handle, without the Python object around it (0.1 against
# 2.6 us).  One request's step, calls in a row: 9.2 us before, 6.5 us so.
def _ptr(t, name, dtype=None):
    if t is None:
        return None
    if (isinstance(t, torch.Tensor) and t.is_cuda and (dtype is None or t.dtype is dtype)
            and t.is_contiguous()):
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _stream(stream):
    if stream is None:  # the current stream of the current device
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return getattr(stream, "cuda_stream", stream)


# (ctypes keeps the low 32 bits of a larger number and says nothing: what a caller
# gives as a number is compared with this, not what a tensor's memory bounds)
_I32 = 2 ** 31 - 1


def make_dims(B, Hq, Hkv, d, L, f, dtype, n_slots, flags=0) -> Dims:
    if not -_I32 <= L <= _I32:
        raise ValueError(f"a block of {L} tokens is not supported")
    return Dims(B, Hq, Hkv, d, L, f, dtype, n_slots, flags)


def _out_flags(out, act, out_f32):
    """Output dtype: fp32 when asked (or when out is an fp32 tensor)."""
    if out is not None:
        out_f32 = out.dtype == torch.float32
    odt = torch.float32 if out_f32 else act
    return (HYB_OUT_F32 if out_f32 and act != torch.float32 else 0), odt


def hybrid_attn_step(q, k, v, W, alpha, S, z, slots=None, out=None, out_f32=False,
                     stream=None, block_len=None, kernel=None):
    """q [B][L][Hq][d], k/v [B][L][Hkv][d], W [Hq][F][d], alpha [Hq] f32,
    S [n_slots][Hq][d][f] f32 (S_h transposed), z [n_slots][Hq][f] f32 -> out [B][L][Hq][d]
    in q's dtype (fp32 with out_f32).  block_len [B] int32 (device): active rows
    per request; rows past it of out are left as they were.  kernel: None or
    "auto" (the library picks), "split", "whole" or "halves" (HYB_STEP_SPLIT /
    HYB_STEP_WHOLE / HYB_STEP_HALVES)."""
    lib = load()
    B, L, Hq, d = q.shape
    act = q.dtype
    flags, odt = _out_flags(out, act, out_f32)
    flags |= _STEP_KERNEL[kernel]
    dims = make_dims(B, Hq, k.shape[2], d, L, z.shape[2], _dt(q), S.shape[0], flags)
    if out is None:
        out = torch.empty(q.shape, dtype=odt, device=q.device)
    _check(lib.hybrid_attn_step(
        ctypes.byref(dims), _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(W, "W", act), _ptr(alpha, "alpha", torch.float32),
        _ptr(S, "S", torch.float32), _ptr(z, "z", torch.float32),
        _ptr(slots, "slots", torch.int32), _ptr(block_len, "block_len", torch.int32),
        _ptr(out, "out", odt), _stream(stream)))
    return out


def hybrid_attn_step_commit(q, k, v, W, alpha, S, z, slots=None, out=None, out_f32=False,
                            stream=None, block_len=None):
    """The step of hybrid_attn_step on the state as it is, then the commit of
    k/v into S, z in place, in one launch; returns out."""
    lib = load()
    B, L, Hq, d = q.shape
    act = q.dtype
    flags, odt = _out_flags(out, act, out_f32)
    dims = make_dims(B, Hq, k.shape[2], d, L, z.shape[2], _dt(q), S.shape[0], flags)
    if out is None:
        out = torch.empty(q.shape, dtype=odt, device=q.device)
    _check(lib.hybrid_attn_step_commit(
        ctypes.byref(dims), _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(W, "W", act), _ptr(alpha, "alpha", torch.float32),
        _ptr(S, "S", torch.float32), _ptr(z, "z", torch.float32),
        _ptr(slots, "slots", torch.int32), _ptr(block_len, "block_len", torch.int32),
        _ptr(out, "out", odt), _stream(stream)))
    return out


def hybrid_state_commit(k, v, W, S, z, slots=None, stream=None, block_len=None):
    """Folds the block k/v [B][L][Hkv][d] into S, z in place."""
    lib = load()
    B, L, Hkv, d = k.shape
    dims = make_dims(B, W.shape[0], Hkv, d, L, z.shape[2], _dt(k), S.shape[0])
    act = k.dtype
    _check(lib.hybrid_state_commit(
        ctypes.byref(dims), _ptr(k, "k"), _ptr(v, "v", act), _ptr(W, "W", act),
        _ptr(S, "S", torch.float32), _ptr(z, "z", torch.float32),
        _ptr(slots, "slots", torch.int32), _ptr(block_len, "block_len", torch.int32),
        _stream(stream)))


def workspace_bytes(dims: Dims, op: int, extent: int = 0) -> int:
    return int(load().hybrid_workspace_bytes(ctypes.byref(dims), op, extent))


def hybrid_state_prefill(q, k, v, W, alpha, S, z, block, slots=None, out=None,
                         want_out=True, out_f32=False, ws=None, stream=None):
    """Block-causal prefill of k/v [B][T][Hkv][d] (and q [B][T][Hq][d] when
    outputs are wanted); updates S, z in place and returns out (or None)."""
    lib = load()
    B, T, Hkv, d = k.shape
    Hq = W.shape[0]
    act = k.dtype
    flags, odt = _out_flags(out, act, out_f32)
    dims = make_dims(B, Hq, Hkv, d, block, z.shape[2], _dt(k), S.shape[0], flags)
    if want_out and out is None:
        out = torch.empty((B, T, Hq, d), dtype=odt, device=k.device)
    if not want_out:
        out = None
    need = workspace_bytes(dims, OP_PREFILL, T)
    if need and ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=k.device)
    _check(lib.hybrid_state_prefill(
        ctypes.byref(dims), T, _ptr(q, "q", act) if want_out else None,
        _ptr(k, "k"), _ptr(v, "v", act), _ptr(W, "W", act),
        _ptr(alpha, "alpha", torch.float32) if want_out else None,
        _ptr(S, "S", torch.float32), _ptr(z, "z", torch.float32),
        _ptr(slots, "slots", torch.int32), _ptr(out, "out", odt) if want_out else None,
        _ptr(ws, "ws") if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return out


def hybrid_state_prefill_noalloc(q, k, v, W, alpha, S, z, block, slots=None, out=None,
                                 want_out=True, out_f32=False, stream=None):
    """hybrid_state_prefill with the library-held scratch buffer as its
    workspace: the call allocates no device memory (out is allocated here
    only when the caller passes none)."""
    lib = load()
    B, T, Hkv, d = k.shape
    Hq = W.shape[0]
    act = k.dtype
    flags, odt = _out_flags(out, act, out_f32)
    dims = make_dims(B, Hq, Hkv, d, block, z.shape[2], _dt(k), S.shape[0], flags)
    if want_out and out is None:
        out = torch.empty((B, T, Hq, d), dtype=odt, device=k.device)
    if not want_out:
        out = None
    _check(lib.hybrid_state_prefill_noalloc(
        ctypes.byref(dims), T, _ptr(q, "q", act) if want_out else None,
        _ptr(k, "k"), _ptr(v, "v", act), _ptr(W, "W", act),
        _ptr(alpha, "alpha", torch.float32) if want_out else None,
        _ptr(S, "S", torch.float32), _ptr(z, "z", torch.float32),
        _ptr(slots, "slots", torch.int32), _ptr(out, "out", odt) if want_out else None,
        _stream(stream)))
    return out


def softmax_prefix_step(q, k, v, k_cache, v_cache, prefix_len, out=None, ws=None,
                        out_f32=False, stream=None):
    """Exact softmax of q [B][L][Hq][d] over k_cache/v_cache [B][Pmax][Hkv][d]
    (first prefix_len[b] rows, int32 on the device) plus the block k/v."""
    lib = load()
    B, L, Hq, d = q.shape
    Hkv = k.shape[2]
    Pmax = k_cache.shape[1]
    act = q.dtype
    flags, odt = _out_flags(out, act, out_f32)
    dims = make_dims(B, Hq, Hkv, d, L, 64, _dt(q), 1, flags)
    if out is None:
        out = torch.empty(q.shape, dtype=odt, device=q.device)
    need = workspace_bytes(dims, OP_SOFTMAX_PREFIX, Pmax)
    if need and ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.softmax_prefix_step(
        ctypes.byref(dims), _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(k_cache, "k_cache", act), _ptr(v_cache, "v_cache", act),
        _ptr(prefix_len, "prefix_len", torch.int32), Pmax, _ptr(out, "out", odt),
        _ptr(ws, "ws") if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return out


def softmax_prefix_step_paged(q, k, v, k_pages, v_pages, page_table, prefix_len, out=None,
                              ws=None, out_f32=False, stream=None):
    """softmax_prefix_step over a paged cache: k_pages/v_pages
    [n_pages][page_size][Hkv][d], page_table [B][max_pages] int32 and
    prefix_len [B] int32 on the device."""
    lib = load()
    B, L, Hq, d = q.shape
    Hkv = k.shape[2]
    n_pages, page_size = k_pages.shape[0], k_pages.shape[1]
    max_pages = min(page_table.shape[1], _I32)
    act = q.dtype
    flags, odt = _out_flags(out, act, out_f32)
    dims = make_dims(B, Hq, Hkv, d, L, 64, _dt(q), 1, flags)
    if out is None:
        out = torch.empty(q.shape, dtype=odt, device=q.device)
    need = workspace_bytes(dims, OP_SOFTMAX_PREFIX, min(max_pages * page_size, _I32))
    if need and ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.softmax_prefix_step_paged(
        ctypes.byref(dims), _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(k_pages, "k_pages", act), _ptr(v_pages, "v_pages", act), n_pages, page_size,
        _ptr(page_table, "page_table", torch.int32), max_pages,
        _ptr(prefix_len, "prefix_len", torch.int32), _ptr(out, "out", odt),
        _ptr(ws, "ws") if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return out


def hybrid_attn_backward(q, k, v, W, alpha, block, dout=None, target=None, dW=None,
                         dalpha=None, loss=None, ws=None, stream=None):
    """Gradient of the block-causal hybrid layer over q [B][T][Hq][d],
    k/v [B][T][Hkv][d] (empty starting state, blocks of `block` tokens) with
    respect to W [Hq][F][d] and alpha [Hq].  Give dout (upstream gradient) or
    target (the teacher's output; squared-error loss).  Returns
    (dW fp32 [Hq][F][d], dalpha fp32 [Hq], loss fp32 [Hq] or None)."""
    lib = load()
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    F = W.shape[1]
    act = q.dtype
    dims = make_dims(B, Hq, Hkv, d, block, 2 * F, _dt(q), 1, 0)
    dev = q.device
    if dW is None:
        dW = torch.empty((Hq, F, d), dtype=torch.float32, device=dev)
    if dalpha is None:
        dalpha = torch.empty(Hq, dtype=torch.float32, device=dev)
    if target is not None and loss is None:
        loss = torch.empty(Hq, dtype=torch.float32, device=dev)
    need = workspace_bytes(dims, OP_BACKWARD, T)
    if ws is None and need:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(lib.hybrid_attn_backward(
        ctypes.byref(dims), T, _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(W, "W", act), _ptr(alpha, "alpha", torch.float32),
        _ptr(dout, "dout", act), _ptr(target, "target", act),
        _ptr(dW, "dW", torch.float32), _ptr(dalpha, "dalpha", torch.float32),
        _ptr(loss, "loss", torch.float32),
        _ptr(ws, "ws") if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return dW, dalpha, loss


def hybrid_attn_backward_full(q, k, v, W, alpha, block, dout=None, target=None, ws=None,
                              stream=None):
    """hybrid_attn_backward plus the gradients with respect to the inputs.
    Returns (dq fp32 [B][T][Hq][d], dk, dv fp32 [B][T][Hkv][d], dW, dalpha,
    loss or None)."""
    lib = load()
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    F = W.shape[1]
    act = q.dtype
    dims = make_dims(B, Hq, Hkv, d, block, 2 * F, _dt(q), 1, 0)
    dev = q.device
    f32 = torch.float32
    dq = torch.empty((B, T, Hq, d), dtype=f32, device=dev)
    dk = torch.empty((B, T, Hkv, d), dtype=f32, device=dev)
    dv = torch.empty((B, T, Hkv, d), dtype=f32, device=dev)
    dW = torch.empty((Hq, F, d), dtype=f32, device=dev)
    dalpha = torch.empty(Hq, dtype=f32, device=dev)
    loss = torch.empty(Hq, dtype=f32, device=dev) if target is not None else None
    need = workspace_bytes(dims, OP_BACKWARD_FULL, T)
    if ws is None and need:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(lib.hybrid_attn_backward_full(
        ctypes.byref(dims), T, _ptr(q, "q"), _ptr(k, "k", act), _ptr(v, "v", act),
        _ptr(W, "W", act), _ptr(alpha, "alpha", f32),
        _ptr(dout, "dout", act), _ptr(target, "target", act),
        _ptr(dq, "dq", f32), _ptr(dk, "dk", f32), _ptr(dv, "dv", f32),
        _ptr(dW, "dW", f32), _ptr(dalpha, "dalpha", f32), _ptr(loss, "loss", f32),
        _ptr(ws, "ws") if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return dq, dk, dv, dW, dalpha, loss


# The entry points below run on the device of their first tensor, whatever the
# current one is, and allocate on the stream they run on, so that a buffer
# made here is neither written before earlier work has left it nor reused
# while the call still runs.
def _placed(f):
    name = list(inspect.signature(f).parameters)[1]

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        try:
            dev = (args[0] if args else kw[name]).get_device()
        except (AttributeError, KeyError):
            dev = -1
        if dev < 0:
            raise TypeError(f"{f.__name__} takes CUDA (HIP) tensors, {name} first")
        if stream is None and dev == torch._C._cuda_getDevice():
            return f(dev, *args, **kw)
        with contextlib.ExitStack() as on:
            on.enter_context(torch.cuda.device(dev))
            if stream is not None:
                if not isinstance(stream, torch.cuda.Stream):  # a raw handle; 0 is the null stream
                    stream = (torch.cuda.ExternalStream(stream, device=dev) if stream
                              else torch.cuda.default_stream(dev))
                if stream.device.index != dev:
                    raise ValueError(f"a stream of {stream.device} for tensors of device {dev}")
                on.enter_context(torch.cuda.stream(stream))
            return f(dev, *args, **kw)
    call.__signature__ = inspect.Signature(
        [p for p in inspect.signature(f).parameters.values() if p.name != "dev"]
        + [inspect.Parameter("stream", inspect.Parameter.KEYWORD_ONLY, default=None)])
    return call


def _dptr(dev, t, name, dtype, shape=None):
    """The address of a contiguous tensor of the device (None for None)."""
    if t is None:
        return None
    try:
        if (t.get_device() == dev and t.dtype is dtype and t.is_contiguous()
                and (shape is None or t.shape == shape)):
            return t.data_ptr()
    except AttributeError:
        pass
    _ptr(t, name, dtype)
    if t.get_device() != dev:
        raise ValueError(f"{name} is on device {t.get_device()}, the call runs on {dev}")
    raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _rows(dev, t, name, dtype, shape):
    """The address and row stride of [N][H][d] whose rows [H][d] are contiguous.
    (A stride of 0, of an expanded tensor, would mean contiguous rows to the library.)"""
    if t is None:
        return None, 0
    try:
        if t.get_device() == dev and t.dtype is dtype and t.shape == shape:
            s = t.stride()
            if s[2] == 1 and (s[1] == shape[2] or shape[1] == 1):
                if shape[0] < 2:  # (a stride says nothing)
                    return t.data_ptr(), 0
                if s[0]:
                    return t.data_ptr(), s[0]
    except AttributeError:
        pass
    _dptr(dev, t.contiguous() if isinstance(t, torch.Tensor) else t, name, dtype, shape)
    raise ValueError(f"{name}: the heads of a token must be contiguous, and the tokens apart")


_CONTIGUOUS = torch.contiguous_format


def _new(t, dtype):
    """A contiguous tensor like t, of dtype."""
    if dtype is t.dtype:
        return torch.empty_like(t, memory_format=_CONTIGUOUS)
    return torch.empty_like(t, dtype=dtype, memory_format=_CONTIGUOUS)


def _ws(dev, t):
    """A workspace's address and size, whatever its type."""
    return (None, 0) if t is None else (_dptr(dev, t, "ws", t.dtype), t.numel() * t.element_size())


# (a ctypes structure costs more to fill than to find; nothing writes to them)
_rope_dims = functools.lru_cache(maxsize=256)(RopeDims)
_dims = functools.lru_cache(maxsize=256)(make_dims)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _odt(act, out, out_f32):
    if out is not None:
        out_f32 = out.dtype == torch.float32
    return torch.float32 if out_f32 else act


def _rope_args(dev, q, k, wq, wk, inv_freq, positions, eps, rot_scale, layout, q_out, k_out, odt,
               v=None, grad=HYB_BF16):
    """Dims and the addresses that the rope entry points share."""
    N, Hq, d = qs = q.shape
    ks = k.shape
    act = q.dtype
    if len(ks) != 3 or ks[0] != N or ks[2] != d:
        raise ValueError(f"k must have shape [{N}][heads][{d}], got {tuple(ks)}")
    pq, sq = _rows(dev, q, "q", act, qs)
    pk, sk = _rows(dev, k, "k", act, ks)
    pv, sv = _rows(dev, v, "v", act, ks)
    oq, soq = _rows(dev, q_out, "q_out", odt, qs)
    ok, sok = _rows(dev, k_out, "k_out", odt, ks)
    dims = _rope_dims(N, Hq, ks[1], d, 2 * inv_freq.shape[0] if inv_freq is not None else 0,
                      _ROPE_LAYOUT[layout], _dt(q), grad,
                      HYB_OUT_F32 if odt is not act else 0, eps, rot_scale, sq, sk, sv, soq, sok)
    return (dims, pq, pk, pv, oq, ok, _dptr(dev, wq, "wq", act, (d,)),
            _dptr(dev, wk, "wk", act, (d,)), _dptr(dev, positions, "positions", torch.int32, (N,)),
            _dptr(dev, inv_freq, "inv_freq", torch.float64, (dims.rot_dim // 2,)))


@_placed
def hybrid_qk_norm_rope(dev, q, k, inv_freq, positions, wq=None, wk=None, eps=1e-6, rot_scale=1.0,
                        layout="half", q_out=None, k_out=None, out_f32=False):
    """Norm (weights wq, wk [d], None: no norm) and rotation of q [N][Hq][d] and
    k [N][Hkv][d], which may be views of one packed projection, by positions [N]
    int32 and inv_freq [rot_dim / 2] float64 (None: no rotation); layout "half"
    or "interleaved".  Returns (q_out, k_out)."""
    odt = _odt(q.dtype, q_out, out_f32)
    if q_out is None:
        q_out = _new(q, odt)
    if k_out is None:
        k_out = _new(k, odt)
    dims, pq, pk, _, oq, ok, pwq, pwk, pos, freq = _rope_args(
        dev, q, k, wq, wk, inv_freq, positions, eps, rot_scale, layout, q_out, k_out, odt)
    _check(load().hybrid_qk_norm_rope(dims, pq, pk, pwq, pwk, pos, freq, oq, ok, _raw_stream(dev)))
    return q_out, k_out


@_placed
def hybrid_qk_norm_rope_paged(dev, q, k, v, inv_freq, positions, slots, k_pages, v_pages, wq=None,
                              wk=None, eps=1e-6, rot_scale=1.0, layout="half", q_out=None,
                              k_out=None, want_k=False, out_f32=False):
    """hybrid_qk_norm_rope with k's result and v [N][Hkv][d] written to rows slots
    [N] (int32; -1: nowhere) of the pools k_pages, v_pages [n_pages][page_size][Hkv][d].
    Returns (q_out, k_out), k_out None unless given or asked for with want_k."""
    odt = _odt(q.dtype, q_out, out_f32)
    if q_out is None:
        q_out = _new(q, odt)
    if k_out is None and want_k:
        k_out = _new(k, odt)
    dims, pq, pk, pv, oq, ok, pwq, pwk, pos, freq = _rope_args(
        dev, q, k, wq, wk, inv_freq, positions, eps, rot_scale, layout, q_out, k_out, odt, v=v)
    n_pages, page_size = k_pages.shape[:2]
    pool = (n_pages, page_size) + tuple(k.shape[1:])
    _check(load().hybrid_qk_norm_rope_paged(
        dims, pq, pk, pv, pwq, pwk, pos, freq,
        _dptr(dev, slots, "slots", torch.int32, (q.shape[0],)), oq, ok,
        _dptr(dev, k_pages, "k_pages", q.dtype, pool),
        _dptr(dev, v_pages, "v_pages", q.dtype, pool), n_pages, page_size, _raw_stream(dev)))
    return q_out, k_out


@_placed
def hybrid_qk_norm_rope_backward(dev, q, k, dq_out, dk_out, inv_freq, positions, wq=None, wk=None,
                                 eps=1e-6, rot_scale=1.0, layout="half", dq=None, dk=None,
                                 out_f32=False, ws=None):
    """Gradient of hybrid_qk_norm_rope for dq_out [N][Hq][d], dk_out [N][Hkv][d]
    (both fp32 or both bf16).  Returns (dq, dk in q's dtype or fp32 with out_f32,
    dwq, dwk fp32 [d] or None where there is no weight)."""
    lib = load()
    odt = _odt(q.dtype, dq, out_f32)
    at, f32, d = q.device, torch.float32, q.shape[2]
    if dq is None:
        dq = _new(q, odt)
    if dk is None:
        dk = _new(k, odt)
    dwq = torch.empty(d, dtype=f32, device=at) if wq is not None else None
    dwk = torch.empty(d, dtype=f32, device=at) if wk is not None else None
    dims, pq, pk, _, oq, ok, pwq, pwk, pos, freq = _rope_args(
        dev, q, k, wq, wk, inv_freq, positions, eps, rot_scale, layout, dq, dk, odt,
        grad=_dt(dq_out))
    if ws is None and (wq is not None or wk is not None):
        ws = torch.empty(lib.hybrid_rope_workspace_bytes(dims), dtype=torch.uint8, device=at)
    _check(lib.hybrid_qk_norm_rope_backward(
        dims, pq, pk, pwq, pwk, pos, freq, _dptr(dev, dq_out, "dq_out", dq_out.dtype, q.shape),
        _dptr(dev, dk_out, "dk_out", dq_out.dtype, k.shape), oq, ok,
        None if dwq is None else dwq.data_ptr(), None if dwk is None else dwk.data_ptr(),
        *_ws(dev, ws), _raw_stream(dev)))
    return dq, dk, dwq, dwk


@_placed
def kv_pages_plan(dev, prefix_len, new_len, page_table, free_pages, page_size, max_tokens):
    """Pages (written into page_table [B][max_pages] int32 from free_pages) and
    rows of the new_len [B] tokens that follow prefix_len [B] cached ones, all
    int32 on the device.  Returns (slots [max_tokens], positions [max_tokens],
    token_start [B + 1], counts [2]: pages taken and missing)."""
    B, max_pages = page_table.shape
    i32, at = torch.int32, prefix_len.device
    if not (0 <= max_tokens <= _I32 and -_I32 <= page_size <= _I32 and max_pages <= _I32):
        raise ValueError(f"max_tokens {max_tokens}, page_size {page_size} and a table of {max_pages} "
                         "pages per request must be 0 .. 2^31 - 1")
    if B == 0:
        return (torch.full((max_tokens,), -1, dtype=i32, device=at),
                *(torch.zeros(n, dtype=i32, device=at) for n in (max_tokens, 1, 2)))
    lens = _dptr(dev, prefix_len, "prefix_len", i32, (B,))
    slots, positions, start, counts = map(prefix_len.new_empty, (max_tokens, max_tokens, B + 1, 2))
    _check(load().kv_pages_plan(
        B, max_pages, page_size, min(free_pages.numel(), _I32) if free_pages is not None else 0,
        max_tokens,
        lens, _dptr(dev, new_len, "new_len", i32, (B,)),
        _dptr(dev, free_pages, "free_pages", i32), _dptr(dev, page_table, "page_table", i32),
        slots.data_ptr(), positions.data_ptr(), start.data_ptr(), counts.data_ptr(),
        _raw_stream(dev)))
    return slots, positions, start, counts


def _reach(n):
    """A window or a number of sinks: one past 2^31 - 1 sees what that one sees (the
    library refuses those below 0)."""
    return max(min(operator.index(n), _I32), -1)


def _window_dims(q, k, block, odt):
    B, n, Hq, d = q.shape
    kv = (B, n, k.shape[2], d)
    return _dims(B, Hq, kv[2], d, block, 64, _dt(q), 1, HYB_OUT_F32 if odt is not q.dtype else 0), kv


@_placed
def softmax_window_step_paged(dev, q, k, v, k_pages, v_pages, page_table, prefix_len, window,
                              n_sinks=0, block_len=None, out=None, ws=None, out_f32=False):
    """softmax_prefix_step_paged over the last `window` cached tokens and the
    first n_sinks, plus the block (the first block_len[b] rows of request b;
    rows past it of out are left as they were, zero if out is made here)."""
    lib = load()
    B, L, Hq, d = q.shape
    act, i32 = q.dtype, torch.int32
    odt = _odt(act, out, out_f32)
    dims, kv = _window_dims(q, k, L, odt)
    if out is None:
        new = torch.empty if block_len is None else torch.zeros
        out = new(q.shape, dtype=odt, device=q.device)
    n_pages, page_size = k_pages.shape[:2]
    pool = (n_pages, page_size, kv[2], d)
    max_pages = min(page_table.shape[1], _I32)
    window, n_sinks = _reach(window), _reach(n_sinks)
    if ws is None:
        need = lib.hybrid_workspace_bytes(dims, OP_WINDOW_STEP,
                                          min(max_pages * page_size, window + n_sinks + 64, _I32))
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _check(lib.softmax_window_step_paged(
        dims, _dptr(dev, q, "q", act), _dptr(dev, k, "k", act, kv), _dptr(dev, v, "v", act, kv),
        _dptr(dev, k_pages, "k_pages", act, pool), _dptr(dev, v_pages, "v_pages", act, pool),
        n_pages, page_size, _dptr(dev, page_table, "page_table", i32, (B, max_pages)), max_pages,
        _dptr(dev, prefix_len, "prefix_len", i32, (B,)), window, n_sinks,
        _dptr(dev, block_len, "block_len", i32, (B,)), _dptr(dev, out, "out", odt, q.shape),
        *_ws(dev, ws), _raw_stream(dev)))
    return out


@_placed
def softmax_window_prefill(dev, q, k, v, block, window, n_sinks=0, seq_lens=None, out=None,
                           lse=None, want_lse=True, ws=None, out_f32=False):
    """Softmax of q [B][T][Hq][d] over k, v [B][T][Hkv][d], block-causal in blocks
    of `block` tokens, over the block, the `window` tokens before it and the
    first n_sinks (a window of T or more: every earlier block).  seq_lens [B]
    int32 (device): rows past them of out and lse are left as they were (zero if
    made here).  Returns (out, lse fp32 [B][Hq][T] or None)."""
    lib = load()
    B, T, Hq, d = q.shape
    act, f32 = q.dtype, torch.float32
    odt = _odt(act, out, out_f32)
    dims, kv = _window_dims(q, k, block, odt)
    window, n_sinks = _reach(window), _reach(n_sinks)
    new = torch.empty if seq_lens is None else torch.zeros
    if out is None:
        out = new(q.shape, dtype=odt, device=q.device)
    if lse is None and want_lse:
        lse = new((B, Hq, T), dtype=f32, device=q.device)
    if ws is None:
        need = lib.hybrid_workspace_bytes(dims, OP_WINDOW_PREFILL, T)
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _check(lib.softmax_window_prefill(
        dims, T, window, n_sinks, _dptr(dev, q, "q", act), _dptr(dev, k, "k", act, kv),
        _dptr(dev, v, "v", act, kv), _dptr(dev, seq_lens, "seq_lens", torch.int32, (B,)),
        _dptr(dev, out, "out", odt, q.shape), _dptr(dev, lse, "lse", f32, (B, Hq, T)),
        *_ws(dev, ws), _raw_stream(dev)))
    return out, lse


@_placed
def softmax_window_backward(dev, q, k, v, out, lse, dout, block, window, n_sinks=0, seq_lens=None,
                            dq=None, dk=None, dv=None, ws=None, out_f32=False):
    """Gradient of softmax_window_prefill for the upstream gradient dout; out (in
    q's dtype) and lse as the forward call left them.  Returns (dq, dk, dv) in
    q's dtype (fp32 with out_f32); rows past seq_lens are zero."""
    lib = load()
    B, T, Hq, d = q.shape
    act, at = q.dtype, q.device
    odt = _odt(act, dq, out_f32)
    dims, kv = _window_dims(q, k, block, odt)
    window, n_sinks = _reach(window), _reach(n_sinks)
    dq = _new(q, odt) if dq is None else dq
    dk = _new(k, odt) if dk is None else dk
    dv = _new(v, odt) if dv is None else dv
    if ws is None:
        need = lib.hybrid_workspace_bytes(dims, OP_WINDOW_BACKWARD, T)
        ws = torch.empty(need, dtype=torch.uint8, device=at)
    _check(lib.softmax_window_backward(
        dims, T, window, n_sinks, _dptr(dev, q, "q", act), _dptr(dev, k, "k", act, kv),
        _dptr(dev, v, "v", act, kv), _dptr(dev, seq_lens, "seq_lens", torch.int32, (B,)),
        _dptr(dev, out, "out", act, q.shape),
        _dptr(dev, lse, "lse", torch.float32, (B, Hq, T)),
        _dptr(dev, dout, "dout", act, q.shape), _dptr(dev, dq, "dq", odt, q.shape),
        _dptr(dev, dk, "dk", odt, kv), _dptr(dev, dv, "dv", odt, kv),
        *_ws(dev, ws), _raw_stream(dev)))
    return dq, dk, dv


_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _q8_pools(dev, k_pages, v_pages, k_scales, v_scales, Hkv, d):
    """The addresses of an 8-bit cache's pools, its pages, their size and the scale block."""
    pool = k_pages.shape
    if len(pool) != 4 or pool[2] != Hkv or pool[3] != d:
        raise ValueError(f"k_pages must have shape [pages][page_size][{Hkv}][{d}], got {tuple(pool)}")
    n_pages, page = pool[0], pool[1]
    blocks = k_scales.shape[1] if k_scales.dim() == 3 else 0
    if blocks < 1 or page % blocks:
        raise ValueError(f"k_scales must have shape [{n_pages}][page_size / scale_block][{Hkv}], got "
                         f"{tuple(k_scales.shape)} for pages of {page}")
    scale = (n_pages, blocks, Hkv)
    return (_dptr(dev, k_pages, "k_pages", _E4M3), _dptr(dev, v_pages, "v_pages", _E4M3, pool),
            _dptr(dev, k_scales, "k_scales", _E8M0, scale),
            _dptr(dev, v_scales, "v_scales", _E8M0, scale)), n_pages, page, page // blocks


_q8_dims = functools.lru_cache(maxsize=256)(KvQ8Dims)


def _q8_args(dev, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first, token_start):
    N, Hkv, d = shape = k.shape
    B, max_pages = page_table.shape
    i32 = torch.int32
    pools, n_pages, page, sb = _q8_pools(dev, k_pages, v_pages, k_scales, v_scales, Hkv, d)
    pk, sk = _rows(dev, k, "k", k.dtype, shape)
    pv, sv = _rows(dev, v, "v", k.dtype, shape)
    dims = _q8_dims(min(N, _I32), B, Hkv, d, _dt(k), min(max_pages, _I32), n_pages, page, sb, sk, sv)
    return dims, pk, pv, pools, (_dptr(dev, page_table, "page_table", i32), _dptr(dev, first, "first", i32, (B,)),
                                 _dptr(dev, token_start, "token_start", i32, (B + 1,)))


@_placed
def kv_pages_q8_write(dev, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first, token_start):
    """Quantises k, v [N][Hkv][d] (views of one packed projection or not) into an
    8-bit cache: k_pages, v_pages [n_pages][page_size][Hkv][d] float8_e4m3fn, k_scales, v_scales
    [n_pages][page_size / scale_block][Hkv] float8_e8m0fnu.  Rows token_start[b] ..
    token_start[b + 1] - 1 (token_start [B + 1] as kv_pages_plan gives it) become tokens
    first[b] .. of request b, whose pages page_table [B][max_pages] names; all int32."""
    dims, pk, pv, pools, where = _q8_args(dev, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first,
                                          token_start)
    _check(load().kv_pages_q8_write(dims, pk, pv, *pools, *where, _raw_stream(dev)))


@_placed
def kv_pages_q8_read(dev, k_pages, v_pages, k_scales, v_scales, page_table, first, token_start, tokens=None,
                     k=None, v=None, dtype=torch.bfloat16):
    """The values of cached tokens first[b] .. of every request as rows token_start[b] ..
    token_start[b + 1] - 1 of k, v [tokens][Hkv][d]; rows without a token are left as they
    were (zero where k or v is made here, in dtype).  Returns (k, v)."""
    given = k if k is not None else v
    if given is None:
        if tokens is None:
            raise TypeError("kv_pages_q8_read needs tokens, the number of rows, or k and v")
        shape, act = (tokens, *k_pages.shape[2:]), dtype
    else:
        shape, act = given.shape, given.dtype
    if k is None:
        k = torch.zeros(shape, dtype=act, device=k_pages.device)
    if v is None:
        v = torch.zeros(shape, dtype=act, device=k_pages.device)
    dims, pk, pv, pools, where = _q8_args(dev, k, v, k_pages, v_pages, k_scales, v_scales, page_table, first,
                                          token_start)
    _check(load().kv_pages_q8_read(dims, *pools, *where, pk, pv, _raw_stream(dev)))
    return k, v


@_placed
def softmax_window_step_paged_q8(dev, q, k, v, k_pages, v_pages, k_scales, v_scales, page_table, prefix_len,
                                 window, n_sinks=0, block_len=None, out=None, ws=None, out_f32=False):
    """softmax_window_step_paged over an 8-bit cache (kv_pages_q8_write); a window of the
    whole prefix or more sees all of it."""
    lib = load()
    B, L, Hq, d = q.shape
    act, i32 = q.dtype, torch.int32
    odt = _odt(act, out, out_f32)
    dims, kv = _window_dims(q, k, L, odt)
    if out is None:
        new = torch.empty if block_len is None else torch.zeros
        out = new(q.shape, dtype=odt, device=q.device)
    pools, n_pages, page, sb = _q8_pools(dev, k_pages, v_pages, k_scales, v_scales, kv[2], d)
    max_pages = min(page_table.shape[1], _I32)
    window, n_sinks = _reach(window), _reach(n_sinks)
    if ws is None:
        need = lib.hybrid_workspace_bytes(dims, OP_WINDOW_STEP_Q8,
                                          min(max_pages * page, window + n_sinks + 64, _I32))
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _check(lib.softmax_window_step_paged_q8(
        dims, _dptr(dev, q, "q", act), _dptr(dev, k, "k", act, kv), _dptr(dev, v, "v", act, kv), *pools,
        n_pages, page, sb, _dptr(dev, page_table, "page_table", i32, (B, max_pages)), max_pages,
        _dptr(dev, prefix_len, "prefix_len", i32, (B,)), window, n_sinks,
        _dptr(dev, block_len, "block_len", i32, (B,)), _dptr(dev, out, "out", odt, q.shape),
        *_ws(dev, ws), _raw_stream(dev)))
    return out


def _packed_args(dev, q, k, v, token_start, block, odt):
    """Dims and the addresses and strides of packed q, k, v, and where the sequences start."""
    N, Hq, d = q.shape
    kv = (N, k.shape[1], d)
    pq, sq = _rows(dev, q, "q", q.dtype, q.shape)
    pk, sk = _rows(dev, k, "k", q.dtype, kv)
    pv, sv = _rows(dev, v, "v", q.dtype, kv)
    dims = _dims(token_start.numel() - 1, Hq, kv[1], d, block, 64, _dt(q), 1,
                 HYB_OUT_F32 if odt is not q.dtype else 0)
    return dims, kv, (pq, pk, pv, sq, sk, sv, _dptr(dev, token_start, "token_start", torch.int32))


@_placed
def softmax_packed_prefill(dev, q, k, v, token_start, block, window, n_sinks=0, out=None, lse=None,
                           want_lse=True, out_f32=False):
    """softmax_window_prefill over packed sequences: rows token_start[b] .. token_start[b + 1]
    - 1 ([B + 1] int32 on the device) of q [N][Hq][d] and k, v [N][Hkv][d], which may be views of
    one packed projection.  block 1 is causal attention, a window of N or more sees every
    earlier block.  Rows behind the last sequence of out and lse are left as they were (zero if
    made here).  Returns (out, lse fp32 [Hq][N] or None)."""
    odt, f32 = _odt(q.dtype, out, out_f32), torch.float32
    N, Hq, _ = q.shape
    dims, _, at = _packed_args(dev, q, k, v, token_start, block, odt)
    if out is None:
        out = torch.zeros(q.shape, dtype=odt, device=q.device)
    if lse is None and want_lse:
        lse = torch.zeros((Hq, N), dtype=f32, device=q.device)
    _check(load().softmax_packed_prefill(
        dims, min(N, _I32), _reach(window), _reach(n_sinks), *at, _dptr(dev, out, "out", odt, q.shape),
        _dptr(dev, lse, "lse", f32, (Hq, N)), _raw_stream(dev)))
    return out, lse


@_placed
def softmax_packed_backward(dev, q, k, v, token_start, out, lse, dout, block, window, n_sinks=0, dq=None,
                            dk=None, dv=None, ws=None, out_f32=False):
    """Gradient of softmax_packed_prefill for the upstream gradient dout; out (in q's dtype)
    and lse as the forward call left them.  Returns (dq, dk, dv) in q's dtype (fp32 with
    out_f32); rows behind the last sequence are zero."""
    lib = load()
    act, odt = q.dtype, _odt(q.dtype, dq, out_f32)
    N, Hq, _ = q.shape
    dims, kv, at = _packed_args(dev, q, k, v, token_start, block, odt)
    dq = _new(q, odt) if dq is None else dq
    dk = _new(k, odt) if dk is None else dk
    dv = _new(v, odt) if dv is None else dv
    if dims.batch == 0:  # no sequence: every row is behind the last
        return dq.zero_(), dk.zero_(), dv.zero_()
    if ws is None and N > 0:
        need = lib.hybrid_workspace_bytes(dims, OP_PACKED_BACKWARD, min(N, _I32))
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.softmax_packed_backward(
        dims, min(N, _I32), _reach(window), _reach(n_sinks), *at, _dptr(dev, out, "out", act, q.shape),
        _dptr(dev, lse, "lse", torch.float32, (Hq, N)), _dptr(dev, dout, "dout", act, q.shape),
        _dptr(dev, dq, "dq", odt, q.shape), _dptr(dev, dk, "dk", odt, kv), _dptr(dev, dv, "dv", odt, kv),
        *_ws(dev, ws), _raw_stream(dev)))
    return dq, dk, dv
