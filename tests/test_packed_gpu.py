"""softmax_packed_prefill and its gradient against 64 bits, a sequence at a time: no token
sees another sequence's, and rows behind the last sequence play no part."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import F32, assert_within, attend, gradient, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32
ALL = 2 ** 31 - 1


def make(lens, Hq, Hkv, d, dtype, seed, tail=0, views=True):
    """q, k, v as views of one projection's rows (or each on its own), NaN behind the last sequence."""
    g = torch.Generator().manual_seed(seed)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n, N = int(start[-1]), int(start[-1]) + tail
    x = torch.randn(N, (Hq + 2 * Hkv) * d, generator=g).to(dtype)
    x[n:] = float("nan")
    x = x.cuda()
    c = {m: x[:, a * d:b * d].unflatten(1, (b - a, d)) for m, a, b in
         (("q", 0, Hq), ("k", Hq, Hq + Hkv), ("v", Hq + Hkv, Hq + 2 * Hkv))}
    if not views:
        c = {m: t.contiguous() for m, t in c.items()}
    dout = torch.randn(N, Hq, d, generator=g)
    dout[n:] = float("nan")
    return dict(c, dout=dout.to(dtype).cuda(), start=torch.from_numpy(start).cuda(), at=start.tolist(), n=n)


def head(c, name, a, b, h):
    return rows64(c[name][a:b, h])


def check_prefill(c, L, window, sinks, out, lse, what=""):
    (_, Hq, _), Hkv = c["q"].shape, c["k"].shape[1]
    bf16 = c["q"].dtype == BF
    for a, b in zip(c["at"], c["at"][1:]):
        if a == b:
            continue
        mask = seen_mask(b - a, L, window, sinks)
        for h in range(Hq):
            g = h * Hkv // Hq
            o, e, oerr, eerr = attend(head(c, "q", a, b, h), head(c, "k", a, b, g), head(c, "v", a, b, g), mask, bf16)
            assert_within(out[a:b, h], o, oerr, out.dtype, f"{what} out {a} h={h}")
            assert_within(lse[h, a:b], e, eerr, FL, f"{what} lse {a} h={h}")


def check_backward(c, L, window, sinks, out, lse, grads, what=""):
    (_, Hq, _), Hkv = c["q"].shape, c["k"].shape[1]
    G, bf16 = Hq // Hkv, c["q"].dtype == BF
    dq, dk, dv = grads
    assert not any(x[c["n"]:].any() for x in grads), "rows behind the last sequence are not zero"
    for a, b in zip(c["at"], c["at"][1:]):
        if a == b:
            continue
        mask = seen_mask(b - a, L, window, sinks)
        for g in range(Hkv):
            sums = [0.0] * 4
            for h in range(g * G, g * G + G):
                r, e = gradient(head(c, "q", a, b, h), head(c, "k", a, b, g), head(c, "v", a, b, g), rows64(out[a:b, h]),
                                rows64(lse[h, a:b]), head(c, "dout", a, b, h), mask, bf16)
                assert_within(dq[a:b, h], r[0], e[0], dq.dtype, f"{what} dq {a} h={h}")
                for i, x in enumerate((r[1], e[1], r[2], e[2])):
                    sums[i] = sums[i] + x
            assert_within(dk[a:b, g], sums[0], sums[1], dk.dtype, f"{what} dk {a} g={g}")
            assert_within(dv[a:b, g], sums[2], sums[3], dv.dtype, f"{what} dv {a} g={g}")


CASES = [  # lens, Hq, Hkv, d, L, window, sinks, dtype, tail
    ([1], 1, 1, 64, 1, ALL, 0, BF, 0),
    ([1, 1, 1, 2, 31, 32, 33, 1], 4, 1, 128, 1, ALL, 0, BF, 3),
    ([0, 5, 0, 0, 64, 127, 0], 8, 2, 64, 1, ALL, 0, BF, 0),
    ([300, 1, 129, 40], 16, 4, 128, 32, ALL, 0, BF, 33),
    ([97, 255, 16], 16, 4, 128, 1, ALL, 0, BF, 0),
    ([200, 340, 7], 8, 8, 64, 16, 40, 5, BF, 1),
    ([511, 3, 260], 4, 2, 64, 1, 100, 130, BF, 0),
    ([70, 150], 12, 4, 128, 21, 33, 0, BF, 0),
    ([90, 35, 1, 64], 10, 2, 64, 7, 0, 0, BF, 5),
    ([65, 130], 16, 1, 64, 1, ALL, 0, BF, 0),            # 16 query heads per KV head
    ([40, 100], 24, 1, 128, 32, 64, 3, BF, 2),           # 24
    ([1, 33, 0, 150], 8, 4, 64, 1, ALL, 0, FL, 7),
    ([130, 64, 5], 4, 2, 128, 32, ALL, 0, FL, 0),
    ([100, 77], 6, 1, 64, 9, 20, 3, FL, 0),
    ([60], 3, 3, 128, 1, 15, 0, FL, 1)]
LONG = [
    ([1500, 20, 700], 4, 1, 64, 1, ALL, 0, BF, 0),       # halves, parts
    ([1200], 8, 2, 128, 32, ALL, 0, BF, 9),
    ([3, 1300, 2, 1100], 2, 1, 128, 1, 300, 200, BF, 0),
    ([20] * 60 + [900], 8, 2, 64, 1, ALL, 0, BF, 0),
    ([900, 5], 4, 1, 128, 1, ALL, 0, FL, 0),
    ([700, 600], 4, 4, 64, 32, 200, 64, FL, 3),
    ([701, 1, 300, 33, 257], 8, 4, 64, 1, ALL, 0, FL, 13),  # few units: a workgroup each
    ([600], 12, 4, 64, 7, ALL, 0, FL, 0),
    ([300, 140, 1], 6, 2, 128, 5, ALL, 3, FL, 4),
    ([520, 31], 4, 4, 128, 1, 300, 40, FL, 1),
    ([500, 480], 3, 1, 64, 1, 100, 170, FL, 2),
    ([125], 16, 2, 128, 1, ALL, 4, FL, 0)]                   # 16 parts


@pytest.mark.parametrize("case,views", [(c, True) for c in CASES + LONG] + [(c, False) for c in CASES], ids=str)
def test_packed(case, views):
    announce(f"packed {case} {views}")
    lens, Hq, Hkv, d, L, window, sinks, dtype, tail = case
    c = make(lens, Hq, Hkv, d, dtype, sum(lens) + L, tail, views)
    args = c["q"], c["k"], c["v"], c["start"]
    N = c["q"].shape[0]
    for f32 in ([False, True] if dtype == BF else [False]):
        out = torch.full((N, Hq, d), 9.0, dtype=FL if f32 else dtype, device="cuda")
        lse = torch.full((Hq, N), 9.0, device="cuda")
        hb.softmax_packed_prefill(*args, L, window, sinks, out=out, lse=lse)
        torch.cuda.synchronize()
        assert bool((out[c["n"]:] == 9.0).all()) and bool((lse[:, c["n"]:] == 9.0).all()), "rows behind were written"
        check_prefill(c, L, window, sinks, out, lse)
    out, lse = hb.softmax_packed_prefill(*args, L, window, sinks)
    out[c["n"]:] = float("nan")
    lse[:, c["n"]:] = float("nan")
    for f32 in ([False, True] if dtype == BF else [False]):
        call = lambda: hb.softmax_packed_backward(*args, out, lse, c["dout"], L, window, sinks, out_f32=f32)
        grads, again = call(), call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(grads, again)), "not the same bits twice"
        check_backward(c, L, window, sinks, out, lse, grads)


def test_many_sequences():
    """More than two looks at 64 starts find, most of them empty or of one token."""
    announce("packed, many sequences")
    r = np.random.RandomState(3)
    lens = r.choice([0, 0, 0, 1, 1, 2], 4500).tolist()
    for i in (0, 64, 4095, 4096, 4499):
        lens[i] = 40 + i % 7
    c = make(lens, 2, 1, 64, BF, 5, 2)
    args = c["q"], c["k"], c["v"], c["start"]
    out, lse = hb.softmax_packed_prefill(*args, 1, ALL)
    grads = hb.softmax_packed_backward(*args, out, lse, c["dout"], 1, ALL)
    torch.cuda.synchronize()
    check_prefill(c, 1, ALL, 0, out, lse)
    check_backward(c, 1, ALL, 0, out, lse, grads)


@pytest.mark.parametrize("dtype,n", [(FL, 260), (BF, 40)])
def test_sequences_past_the_levels(dtype, n):
    """256 sequences and more follow one another instead of going by levels (fp32: a workgroup per unit)."""
    announce(f"packed, 258 sequences {dtype}")
    c = make([n] * 256 + [0, n + 7], 1, 1, 64, dtype, 6, 3)
    args = c["q"], c["k"], c["v"], c["start"]
    out, lse = hb.softmax_packed_prefill(*args, 1, ALL)
    grads = hb.softmax_packed_backward(*args, out, lse, c["dout"], 1, ALL)
    torch.cuda.synchronize()
    check_prefill(c, 1, ALL, 0, out, lse)
    check_backward(c, 1, ALL, 0, out, lse, grads)


def test_as_padded():
    """The padded call of the same sequences: outputs within a rounding each of 64 bits, so
    within two of each other; here, where the order of the sums is the same, equal."""
    announce("packed as padded")
    lens = [200, 31, 170]
    c = make(lens, 8, 2, 128, BF, 7, 0)
    pad = {m: torch.zeros(3, 200, *c[m].shape[1:], dtype=BF, device="cuda") for m in ("q", "k", "v", "dout")}
    for m, t in pad.items():
        for b, (a, e) in enumerate(zip(c["at"], c["at"][1:])):
            t[b, :e - a] = c[m][a:e]
    seq = torch.tensor(lens, dtype=torch.int32).cuda()
    out, lse = hb.softmax_packed_prefill(c["q"], c["k"], c["v"], c["start"], 32, 64, 3)
    po, pl = hb.softmax_window_prefill(pad["q"], pad["k"], pad["v"], 32, 64, 3, seq_lens=seq)
    for b, (a, e) in enumerate(zip(c["at"], c["at"][1:])):
        assert torch.equal(out[a:e], po[b, :e - a]) and torch.equal(lse[:, a:e], pl[b, :, :e - a])


def test_starts_out_of_range():
    """Starts past the rows, below zero and a first that is not zero are clamped."""
    announce("packed, starts out of range")
    c = make([50, 60, 40], 4, 2, 64, BF, 9)
    c["start"].copy_(torch.tensor([-7, 50, 110, 2 ** 31 - 1], dtype=torch.int32))
    args = c["q"], c["k"], c["v"], c["start"]
    out, lse = hb.softmax_packed_prefill(*args, 1, ALL)
    grads = hb.softmax_packed_backward(*args, out, lse, c["dout"], 1, ALL)
    torch.cuda.synchronize()
    check_prefill(c, 1, ALL, 0, out, lse)
    check_backward(c, 1, ALL, 0, out, lse, grads)


def test_nothing():
    """No rows; no sequences: gradients of zero."""
    announce("packed, nothing")
    e = torch.empty(0, 4, 64, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = hb.softmax_packed_prefill(e, e, e, start, 1, ALL)
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    assert all(g.numel() == 0 for g in hb.softmax_packed_backward(e, e, e, start, out, lse, e, 1, ALL))
    x = torch.randn(5, 4, 64, device="cuda")
    out, lse = hb.softmax_packed_prefill(x, x, x, start[:1], 1, ALL)
    assert not out.any()
    assert not any(g.any() for g in hb.softmax_packed_backward(x, x, x, start[:1], out, lse, x, 1, ALL))


def test_gradient_against_differences():
    """fp32: the three gradients along random directions against central differences of
    the 64-bit forward."""
    announce("packed, differences")
    lens, L, window, sinks = [40, 9, 26], 4, 20, 3
    c = make(lens, 4, 2, 64, FL, 11, 0)
    args = c["q"], c["k"], c["v"], c["start"]
    out, lse = hb.softmax_packed_prefill(*args, L, window, sinks)
    grads = hb.softmax_packed_backward(*args, out, lse, c["dout"], L, window, sinks)
    x = {n: rows64(c[n]) for n in ("q", "k", "v")}
    up, rng = rows64(c["dout"]), np.random.default_rng(4)
    t = {n: rng.standard_normal(v.shape) for n, v in x.items()}

    def value(s):
        y = {n: x[n] + s * t[n] for n in x}
        return sum(float((attend(y["q"][a:b, h], y["k"][a:b, h // 2], y["v"][a:b, h // 2],
                                 seen_mask(b - a, L, window, sinks), False)[0] * up[a:b, h]).sum())
                   for a, b in zip(c["at"], c["at"][1:]) for h in range(4))

    h = 1e-5
    want = (value(h) - value(-h)) / (2 * h)
    terms = [rows64(g) * t[n] for g, n in zip(grads, "qkv")]
    have, size = sum(float(a.sum()) for a in terms), sum(float(np.abs(a).sum()) for a in terms)
    # fp32 gradients (about a hundred roundings), and the differences' h^2
    assert abs(want - have) <= size * (400 * F32 + 1e-7), (want, have)


def test_streams_and_replays():
    """Another stream, and a captured forward and gradient that take the starts of each replay."""
    announce("packed, replays")
    c = make([100, 70], 8, 2, 128, BF, 13, 0)
    c["q"], c["k"], c["v"] = (c[m].contiguous() for m in ("q", "k", "v"))
    run = lambda **kw: hb.softmax_packed_prefill(c["q"], c["k"], c["v"], c["start"], 32, 64, 4, **kw)
    back = lambda o, e, **kw: hb.softmax_packed_backward(c["q"], c["k"], c["v"], c["start"], o, e, c["dout"], 32, 64, 4, **kw)
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
    for at in ([0, 100, 170], [0, 0, 170], [0, 33, 90], [0, 100, 170]):
        c["start"].copy_(torch.tensor(at, dtype=torch.int32))
        for x in ("q", "k", "v", "dout"):
            c[x].copy_(torch.randn_like(c[x].float()).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        w = run()
        wb = back(*w)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o + g, w + wb)), at
