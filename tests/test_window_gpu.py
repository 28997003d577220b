"""softmax_window_prefill and softmax_window_backward against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import F32, assert_within, attend, gradient, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def make(B, T, Hq, Hkv, d, dtype, seed, lens=None, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda h: (scale * torch.randn(B, T, h, d, generator=g)).to(dtype).cuda()
    c = dict(q=rnd(Hq), k=rnd(Hkv), v=rnd(Hkv), dout=rnd(Hq), lens=None)
    if lens is not None:
        c["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
        for b, n in enumerate(lens):  # padding may hold anything
            for x in ("q", "k", "v", "dout"):
                c[x][b, min(max(n, 0), T):] = float("nan")
    return c


def lengths(c):
    B, T = c["q"].shape[:2]
    return [T] * B if c["lens"] is None else [min(max(n, 0), T) for n in c["lens"].tolist()]


def heads(c, b, n, h):
    g = h * c["k"].shape[2] // c["q"].shape[2]
    return rows64(c["q"][b, :n, h]), rows64(c["k"][b, :n, g]), rows64(c["v"][b, :n, g])


CASES = [  # B, T, Hq, Hkv, d, L, window, sinks, dtype, lens
    (1, 1, 1, 1, 64, 1, 0, 0, BF, None),
    (1, 33, 4, 1, 128, 1, 5, 2, BF, None),
    (2, 64, 16, 4, 128, 32, 0, 0, BF, None),
    (2, 257, 16, 4, 128, 32, 64, 4, BF, [257, 100]),
    (1, 300, 3, 1, 64, 1, 300, 0, BF, None),
    (3, 197, 8, 4, 64, 21, 50, 5, BF, [197, 0, 21]),
    (1, 500, 5, 5, 64, 32, 100, 33, BF, None),
    (1, 290, 6, 2, 128, 7, 2 ** 31 - 1, 0, BF, None),
    (2, 130, 8, 8, 128, 16, 31, 200, BF, [129, 1]),
    (1, 420, 32, 2, 64, 32, 65, 31, BF, None),
    (1, 611, 4, 4, 128, 32, 2000, 0, BF, None),
    (1, 1, 2, 1, 128, 32, 0, 0, FL, None),
    (2, 197, 8, 4, 64, 21, 50, 5, FL, [197, 64]),
    (1, 130, 4, 2, 128, 32, 1000, 0, FL, None),
    (2, 161, 3, 3, 128, 1, 33, 3, FL, [0, 161]),
    (1, 97, 12, 4, 64, 9, 10, 2 ** 31 - 1, FL, None),
]
IDS = [f"B{c[0]}-T{c[1]}-{c[2]}x{c[3]}-d{c[4]}-L{c[5]}-w{c[6]}-s{c[7]}-{'bf16' if c[8] is BF else 'f32'}" for c in CASES]


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,dtype,lens", CASES, ids=IDS)
def test_prefill(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens):
    announce(f"window prefill {B} {T} {Hq} {Hkv} {d} {L} {window} {sinks} {dtype} {lens}")
    c = make(B, T, Hq, Hkv, d, dtype, T + L, lens)
    for f32 in ([False, True] if dtype == BF else [False]):
        out = torch.full_like(c["q"], 9.0, dtype=FL if f32 else dtype)
        lse = torch.full((B, Hq, T), 9.0, device="cuda")
        hb.softmax_window_prefill(c["q"], c["k"], c["v"], L, window, sinks, seq_lens=c["lens"], out=out, lse=lse)
        torch.cuda.synchronize()
        for b, n in enumerate(lengths(c)):
            assert bool((out[b, n:] == 9.0).all()) and bool((lse[b, :, n:] == 9.0).all()), "padding was written"
            if n == 0:
                continue
            mask = seen_mask(n, L, window, sinks)
            for h in range(Hq):
                o, e, oerr, eerr = attend(*heads(c, b, n, h), mask, dtype == BF)
                assert_within(out[b, :n, h], o, oerr, out.dtype, f"out b={b} h={h}")
                assert_within(lse[b, h, :n], e, eerr, FL, f"lse b={b} h={h}")


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,dtype,lens", CASES, ids=IDS)
def test_backward(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens):
    announce(f"window backward {B} {T} {Hq} {Hkv} {d} {L} {window} {sinks} {dtype} {lens}")
    c = make(B, T, Hq, Hkv, d, dtype, T + L + 1, lens)
    out, lse = hb.softmax_window_prefill(c["q"], c["k"], c["v"], L, window, sinks, seq_lens=c["lens"])
    for b, n in enumerate(lengths(c)):
        out[b, n:] = float("nan")
        lse[b, :, n:] = float("nan")
    call = lambda f32: hb.softmax_window_backward(c["q"], c["k"], c["v"], out, lse, c["dout"], L, window, sinks,
                                                  seq_lens=c["lens"], out_f32=f32)
    for f32 in ([False, True] if dtype == BF else [False]):
        dq, dk, dv = call(f32)
        again = call(f32)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((dq, dk, dv), again)), "not the same bits twice"
        for b, n in enumerate(lengths(c)):
            assert not dq[b, n:].any() and not dk[b, n:].any() and not dv[b, n:].any(), "padding is not zero"
            if n == 0:
                continue
            mask = seen_mask(n, L, window, sinks)
            G = Hq // Hkv
            for g in range(Hkv):
                sums = [0.0] * 4
                for h in range(g * G, g * G + G):
                    r, e = gradient(*heads(c, b, n, h), rows64(out[b, :n, h]), rows64(lse[b, h, :n]),
                                    rows64(c["dout"][b, :n, h]), mask, dtype == BF)
                    assert_within(dq[b, :n, h], r[0], e[0], dq.dtype, f"dq b={b} h={h}")
                    for i, x in enumerate((r[1], e[1], r[2], e[2])):
                        sums[i] = sums[i] + x
                assert_within(dk[b, :n, g], sums[0], sums[1], dk.dtype, f"dk b={b} g={g}")
                assert_within(dv[b, :n, g], sums[2], sums[3], dv.dtype, f"dv b={b} g={g}")


def test_gradient_against_differences():
    """fp32: the three gradients along random directions against central
    differences of the 64-bit forward."""
    B, T, Hq, Hkv, d, L, window, sinks = 1, 75, 4, 2, 64, 8, 20, 3
    c = make(B, T, Hq, Hkv, d, FL, 3)
    out, lse = hb.softmax_window_prefill(c["q"], c["k"], c["v"], L, window, sinks)
    dq, dk, dv = hb.softmax_window_backward(c["q"], c["k"], c["v"], out, lse, c["dout"], L, window, sinks)
    x = {n: rows64(c[n][0]) for n in ("q", "k", "v")}
    up, mask, rng = rows64(c["dout"][0]), seen_mask(T, L, window, sinks), np.random.default_rng(4)
    t = {n: rng.standard_normal(v.shape) for n, v in x.items()}

    def value(s):
        y = {n: x[n] + s * t[n] for n in x}
        return sum(float((attend(y["q"][:, h], y["k"][:, h // 2], y["v"][:, h // 2], mask, False)[0] * up[:, h]).sum())
                   for h in range(Hq))

    h = 1e-5
    want = (value(h) - value(-h)) / (2 * h)
    terms = [rows64(g[0]) * t[n] for g, n in ((dq, "q"), (dk, "k"), (dv, "v"))]
    have = sum(float(a.sum()) for a in terms)
    size = sum(float(np.abs(a).sum()) for a in terms)
    # fp32 gradients (about a hundred roundings), and the differences' h^2
    assert abs(want - have) <= size * (400 * F32 + 1e-7), (want, have)


def test_teacher_of_the_attention_transfer():
    """window >= T is block-causal softmax: what the hybrid layer's gradient
    takes as target; its loss against the layer's own outputs."""
    B, T, Hq, Hkv, d, L = 1, 96, 4, 2, 64, 32
    c = make(B, T, Hq, Hkv, d, FL, 8)
    target, _ = hb.softmax_window_prefill(c["q"], c["k"], c["v"], L, T, want_lse=False)
    g = torch.Generator().manual_seed(1)
    W = (0.1 * torch.randn(Hq, 32, d, generator=g)).cuda()
    alpha = torch.zeros(Hq).cuda()
    S, z = torch.zeros(B, Hq, d, 64, device="cuda"), torch.zeros(B, Hq, 64, device="cuda")
    out = hb.hybrid_state_prefill(c["q"], c["k"], c["v"], W, alpha, S, z, L)
    _, _, loss = hb.hybrid_attn_backward(c["q"], c["k"], c["v"], W, alpha, L, target=target)
    torch.cuda.synchronize()
    want = ((out - target).double() ** 2).sum((0, 1, 3))
    assert float((loss - want).abs().max()) <= 1e-4 * float(want.max())


def test_large_scores():
    """Scores of some hundreds: the running maximum keeps the weights in range."""
    c = make(1, 200, 4, 2, 64, FL, 12, scale=8.0)
    out, lse = hb.softmax_window_prefill(c["q"], c["k"], c["v"], 4, 100, 2)
    mask = seen_mask(200, 4, 100, 2)
    for h in range(4):
        o, e, oerr, eerr = attend(*heads(c, 0, 200, h), mask, False)
        assert_within(out[0, :, h], o, oerr, FL, "out")
        assert_within(lse[0, h], e, eerr, FL, "lse")


def test_streams_and_replays():
    c = make(2, 170, 8, 2, 128, BF, 13, [170, 90])
    run = lambda **kw: hb.softmax_window_prefill(c["q"], c["k"], c["v"], 32, 64, 4, seq_lens=c["lens"], **kw)
    back = lambda o, e, **kw: hb.softmax_window_backward(c["q"], c["k"], c["v"], o, e, c["dout"], 32, 64, 4,
                                                         seq_lens=c["lens"], **kw)
    want = run()
    wb = back(*want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(stream=s)
    gb = back(*got, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + gb, want + wb))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = run()
        g = back(*o)
    for lens in ([170, 90], [3, 170], [0, 64]):
        c["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        for x in ("q", "k", "v", "dout"):
            c[x].copy_(torch.randn_like(c[x].float()).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        w = run()
        wb = back(*w)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o + g, w + wb)), lens


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,dtype,lens", [
    (1, 1500, 4, 1, 64, 1, 100, 3, BF, [1400]), (1, 1000, 8, 2, 128, 32, 1000, 0, BF, None),
    (2, 700, 2, 2, 64, 16, 64, 300, BF, [700, 130]), (1, 900, 6, 1, 128, 8, 31, 150, FL, [890]),
    (1, 1300, 3, 1, 64, 32, 1300, 0, FL, None)])
def test_backward_in_parts(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens):
    """Few keys and many queries: the lists of queries are cut into parts, the
    sinks' into more of them."""
    test_backward(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens)


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,dtype,lens", [
    (1, 1300, 1, 1, 128, 32, 1300, 0, BF, None), (2, 1300, 1, 1, 128, 32, 1300, 200, BF, [1300, 1153]),
    (1, 1290, 1, 1, 64, 1, 1290, 0, BF, None), (1, 1300, 1, 1, 128, 32, 1300, 0, FL, None)])
def test_backward_parts_without_tiles(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens):
    """The last keys are seen by fewer tiles of queries than their list has
    parts: a part that adds nothing leaves zeros."""
    for _ in range(3):
        test_backward(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens)


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks", [
    (1, 40, 4, 4, 64, 1, 3, 0), (2, 1100, 32, 8, 64, 32, 64, 40), (1, 90, 2, 1, 128, 7, 20, 9)])
def test_prefill_f32_halves(B, T, Hq, Hkv, d, L, window, sinks):
    """fp32 with a half of the waves without tiles, and grids past the halves."""
    test_prefill(B, T, Hq, Hkv, d, L, window, sinks, FL, [T - 3 * b for b in range(B)])


@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,lens", [
    (1, 1100, 4, 1, 128, 32, 1100, 0, None), (2, 1057, 2, 1, 64, 1, 1024, 3, [1057, 31]),
    (1, 1090, 3, 3, 64, 32, 64, 1000, [1025]), (2, 1024, 2, 2, 128, 8, 1020, 0, [1, 1024])])
def test_halves(B, T, Hq, Hkv, d, L, window, sinks, lens):
    """Long lists and few workgroups: two halves take a list's tiles in turn,
    one of them without any for the first queries."""
    test_prefill(B, T, Hq, Hkv, d, L, window, sinks, BF, lens)
    test_backward(B, T, Hq, Hkv, d, L, window, sinks, BF, lens)


@pytest.mark.parametrize("B,T,Hq,Hkv,L,window,sinks,lens", [
    (1, 700, 2, 2, 32, 30, 0, [650]), (2, 3001, 2, 1, 1, 511, 4, [3001, 2500]), (4, 290, 4, 2, 16, 290, 0, None),
    (4, 1500, 4, 4, 32, 1500, 0, [1500, 3, 0, 700])])
def test_backward_halves(B, T, Hq, Hkv, L, window, sinks, lens):
    """d = 64: keys' workgroups with and without halves, in one part and in more."""
    test_backward(B, T, Hq, Hkv, 64, L, window, sinks, BF, lens)
