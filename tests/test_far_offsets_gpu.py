"""Norm and rotation, the paged cache and the windowed softmax where offsets
pass 32 bits: the last rows of tensors of more than 2^31 elements."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import BF16, F32, assert_within, attend, gradient, norm_rope, norm_rope_gradient, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def rnd(*shape):
    return torch.empty(shape, dtype=BF, device="cuda").normal_()


def test_rope_rows():
    N, Hq, Hkv, d = 290000, 64, 1, 128
    assert N * Hq * d > 2 ** 31
    announce(f"norm and rotation of {N} x {Hq} heads")
    torch.manual_seed(1)
    q, k = rnd(N, Hq, d), rnd(N, Hkv, d)
    w = 1 + 0.1 * rnd(d)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    freq = torch.logspace(0, -4, d // 2, dtype=torch.float64, device="cuda")
    oq, ok = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq=w, wk=w)
    # (a gradient of zero but for the last rows)
    gq, gk = torch.zeros_like(q), torch.zeros_like(k)
    gq[-5:], gk[-5:] = rnd(5, Hq, d), rnd(5, Hkv, d)
    dq, dk, dwq, dwk = hb.hybrid_qk_norm_rope_backward(q, k, gq, gk, freq, pos, wq=w, wk=w)
    torch.cuda.synchronize()
    for x, y, what in ((q, oq, "q"), (k, ok, "k")):
        ref, mag = norm_rope(rows64(x[-5:]), rows64(w), pos[-5:].cpu().numpy(), rows64(freq), "half", 1e-6, 1.0)
        assert_within(y[-5:], ref, 24 * F32 * mag, BF, what)
    for x, g, dx, dw, what in ((q, gq, dq, dwq, "q"), (k, gk, dk, dwk, "k")):
        rx, rw, ex, ew = norm_rope_gradient(rows64(x[-5:]), rows64(w), rows64(g[-5:]), pos[-5:].cpu().numpy(), rows64(freq),
                                            "half", 1e-6, 1.0)
        assert_within(dx[-5:], rx, ex, BF, "d" + what)
        assert_within(dw, rw, ew, torch.float32, "dw" + what)
        assert not dx[:-5].any()


def test_pages():
    page, Hkv, Hq, d, n = 64, 8, 16, 128, 33000
    assert n * page * Hkv * d > 2 ** 31
    announce(f"pools of {n} pages of {page} x {Hkv} heads")
    torch.manual_seed(2)
    kp, vp = torch.zeros(n, page, Hkv, d, dtype=BF, device="cuda"), torch.zeros(n, page, Hkv, d, dtype=BF, device="cuda")
    table = torch.tensor([[n - 1, 3, n - 2], [1, n - 3, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([150, 110], dtype=torch.int32, device="cuda")
    freq = torch.logspace(0, -4, d // 2, dtype=torch.float64, device="cuda")
    # the cached tokens come by way of the pools' own writer
    cached = []
    for b, m in enumerate(lens.tolist()):
        j = torch.arange(m, device="cuda")
        slots = (table[b][j // page] * page + j % page).to(torch.int32)
        k, v = rnd(m, Hkv, d), rnd(m, Hkv, d)
        _, ko = hb.hybrid_qk_norm_rope_paged(rnd(m, Hq, d), k, v, freq, j.to(torch.int32), slots, kp, vp, want_k=True)
        cached.append((ko, v))
        assert torch.equal(kp.view(-1, Hkv, d)[slots.long()], ko) and torch.equal(vp.view(-1, Hkv, d)[slots.long()], v)
    for L in (1, 8, 32):
        q, k, v = rnd(2, L, Hq, d), rnd(2, L, Hkv, d), rnd(2, L, Hkv, d)
        out = hb.softmax_window_step_paged(q, k, v, kp, vp, table, lens, 70, 5)
        torch.cuda.synchronize()
        for b, m in enumerate(lens.tolist()):
            j = torch.tensor([x for x in range(m) if x >= m - 70 or x < 5], device="cuda")
            kb, vb = (np.concatenate([rows64(c[j]), rows64(x[b])]) for c, x in zip(cached[b], (k, v)))
            for h in range(Hq):
                o, _, err, _ = attend(rows64(q[b, :, h]), kb[:, h // 2], vb[:, h // 2], np.ones((L, len(kb)), bool), True)
                assert_within(out[b, :, h], o, err * 1.001 + BF16 * 1.01 * np.abs(o), BF, f"L={L} b={b} h={h}")


def test_window_rows():
    T, Hq, Hkv, d, window = 270000, 64, 1, 128, 48
    assert T * Hq * d > 2 ** 31
    announce(f"windowed softmax of {T} x {Hq} heads")
    torch.manual_seed(3)
    q, k, v, dout = rnd(1, T, Hq, d), rnd(1, T, Hkv, d), rnd(1, T, Hkv, d), rnd(1, T, Hq, d)
    out, lse = hb.softmax_window_prefill(q, k, v, 1, window)
    dq, dk, dv = hb.softmax_window_backward(q, k, v, out, lse, dout, 1, window)
    torch.cuda.synchronize()
    n = 96  # the last rows: queries of the last 40 see no key before them, and no query before them their keys
    mask = seen_mask(n, 1, window, 0)
    sums = [0.0] * 4
    for h in range(Hq):
        x = rows64(q[0, -n:, h]), rows64(k[0, -n:, 0]), rows64(v[0, -n:, 0])
        o, e, oerr, eerr = attend(*x, mask, True)
        assert_within(out[0, -40:, h], o[-40:], oerr[-40:], BF, f"out h={h}")
        assert_within(lse[0, h, -40:], e[-40:], eerr[-40:], torch.float32, f"lse h={h}")
        r, b = gradient(*x, rows64(out[0, -n:, h]), rows64(lse[0, h, -n:]), rows64(dout[0, -n:, h]), mask, True)
        assert_within(dq[0, -40:, h], r[0][-40:], b[0][-40:], BF, f"dq h={h}")
        for i, y in enumerate((r[1], b[1], r[2], b[2])):
            sums[i] = sums[i] + y
    assert_within(dk[0, -40:, 0], sums[0][-40:], sums[1][-40:], BF, "dk")
    assert_within(dv[0, -40:, 0], sums[2][-40:], sums[3][-40:], BF, "dv")
