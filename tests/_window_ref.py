"""Softmax over a window and the first tokens, and the norm with rotation, in
64 bits on the host, written from the definitions, with the elementwise bounds
the kernels' roundings allow (a bf16 rounding is off by at most 2^-8 of the
value; an fp32 one by 2^-24)."""
from __future__ import annotations

import math

import numpy as np
import torch

BF16, F32 = 2.0 ** -8, 2.0 ** -24


def seen_mask(n, L, window, sinks):
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    s0 = i // L * L
    return (j < s0 + L) & ((j >= s0 - window) | (j < sinks))


def rows64(t):
    return t.detach().double().cpu().numpy()


def score_err(q, k, d):
    """Bound of the error of a scaled score: its d products are summed in fp32,
    and it is scaled and subtracted from its reference there."""
    return F32 * (d + 8) * float((np.abs(q) @ np.abs(k).T).max()) / math.sqrt(d) + 8 * F32


def attend(q, k, v, mask, bf16):
    """q [n, d] over k, v [m, d] -> out, lse and the bounds of their errors
    before a bf16 out is rounded."""
    d = q.shape[1]
    sc = np.where(mask, q @ k.T / math.sqrt(d), -np.inf)
    m = sc.max(1, keepdims=True)
    p = np.exp(sc - m)
    den = p.sum(1, keepdims=True)
    w = p / den
    e = 2 * score_err(q, k, d) + 64 * F32  # of a weight: its own score and the sum's
    rel = e + (1.01 * BF16 if bf16 else 0.0)
    n = mask.sum(1, keepdims=True)
    out_err = (rel + 2 * n * F32) * (w @ np.abs(v))
    lse = (m + np.log(den))[:, 0]
    return w @ v, lse, out_err, e + 8 * F32 * np.abs(lse) + n[:, 0] * F32


def gradient(q, k, v, out, lse, dout, mask, bf16):
    """The gradient as a function of the forward's out and lse as given, and
    the bounds of its errors before the results are rounded."""
    d = q.shape[1]
    sq = 1.0 / math.sqrt(d)
    p = np.where(mask, np.exp(q @ k.T * sq - lse[:, None]), 0.0)
    dp = dout @ v.T
    delta = (dout * out).sum(1, keepdims=True)
    ds = p * (dp - delta)
    e = 2 * score_err(q, k, d) + 64 * F32 + 4 * F32 * np.abs(lse).max()
    # dS: the weight's error on |dP - delta|, and those of the two sums
    ds_err = e * np.abs(ds) + p * d * 2 * F32 * (np.abs(dout) @ np.abs(v).T + (np.abs(dout * out)).sum(1, keepdims=True))
    r = 1.01 * BF16 if bf16 else 0.0
    n = max(mask.shape) * 2 * F32
    dse = ds_err + (r + n) * np.abs(ds)
    return (sq * ds @ k, sq * ds.T @ q, p.T @ dout), (
        sq * dse @ np.abs(k), sq * dse.T @ np.abs(q), ((e + r + n) * p).T @ np.abs(dout))


def assert_within(got, ref, bound, dtype, what):
    """|got - ref| <= bound, plus one rounding where the result is bf16."""
    got = rows64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    tol = bound + (BF16 if dtype == torch.bfloat16 else 4 * F32) * (np.abs(ref) + bound) + 1e-30
    worst = float((np.abs(got - ref) / tol).max()) if got.size else 0.0
    print(f"[parity] {what}: {worst:.3f} of the bound")
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


def norm_rope(x, w, pos, inv_freq, layout, eps, scale):
    """x [N, H, d] -> y, and |a| + |b| of each entry's pair (what its error scales with)."""
    n = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y, mag = n.copy(), np.abs(n)
    rot = 2 * len(inv_freq)
    if rot:
        ang = pos.astype(np.float64)[:, None, None] * inv_freq
        c, s = np.cos(ang) * scale, np.sin(ang) * scale
        ia = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
        ib = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
        a, b = n[..., ia], n[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        mag[..., ia] = mag[..., ib] = (np.abs(a) + np.abs(b)) * abs(scale)
    return y, mag


def norm_rope_gradient(x, w, g, pos, inv_freq, layout, eps, scale):
    """dx, dw and the bounds of their errors before rounding."""
    u, mag = norm_rope(g, None, -pos.astype(np.float64), inv_freq, layout, eps, scale)
    if w is None:
        return u, None, 24 * F32 * mag, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh = x * r
    gn = u * w
    dx = r * (gn - xh * (gn * xh).mean(-1, keepdims=True))
    gm = mag * np.abs(w)
    dx_err = 96 * F32 * r * (gm + np.abs(xh) * (gm * np.abs(xh)).mean(-1, keepdims=True))
    # a sum of n terms in fp32: at most n roundings of the terms' size
    rows = x.shape[0] * x.shape[1]
    dw_err = (64 + min(rows, 512)) * F32 * (mag * np.abs(xh)).sum((0, 1))
    return dx, (u * xh).sum((0, 1)), dx_err, dw_err
