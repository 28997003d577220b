"""hybrid_qk_norm_rope, its paged form and its gradient against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import F32, assert_within, norm_rope, norm_rope_gradient, rows64

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def make(N, Hq, Hkv, d, rot, dtype, seed, norm=True, packed=True, far=1 << 20, gap=0):
    g = torch.Generator().manual_seed(seed)
    width = (Hq + 2 * Hkv) * d + gap
    qkv = (1.5 * torch.randn(N, width, generator=g)).to(dtype).cuda()
    q = qkv[:, :Hq * d].unflatten(1, (Hq, d))
    k = qkv[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
    v = qkv[:, (Hq + Hkv) * d:(Hq + 2 * Hkv) * d].unflatten(1, (Hkv, d))
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos = torch.randint(0, far, (N,), generator=g).to(torch.int32).cuda()
    freq = (1e6 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))).cuda()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    return q, k, v, pos, freq, w[0], w[1]


def ref(x, w, pos, freq, layout, eps=1e-6, scale=1.0):
    y, mag = norm_rope(rows64(x), None if w is None else rows64(w), pos.cpu().numpy(), rows64(freq), layout, eps, scale)
    return y, 24 * F32 * mag


SHAPES = [  # N, Hq, Hkv, d, rot, layout, dtype, norm, packed
    (1, 16, 4, 128, 128, "half", BF, True, True),
    (1, 1, 1, 64, 64, "interleaved", FL, True, False),
    (3, 5, 5, 64, 8, "half", BF, True, True),
    (67, 16, 4, 128, 64, "interleaved", BF, True, True),
    (67, 12, 3, 128, 40, "half", FL, True, True),
    (129, 7, 2, 64, 48, "half", BF, False, False),
    (1031, 8, 4, 64, 64, "half", FL, True, True),
    (2500, 16, 4, 128, 128, "half", BF, True, True),
    (33, 3, 1, 128, 0, "half", BF, True, True),
    (5000, 32, 8, 128, 128, "interleaved", BF, True, True),
]


@pytest.mark.parametrize("N,Hq,Hkv,d,rot,layout,dtype,norm,packed", SHAPES)
@pytest.mark.parametrize("out_f32", [False, True])
def test_forward(N, Hq, Hkv, d, rot, layout, dtype, norm, packed, out_f32):
    announce(f"rope {N} {Hq} {Hkv} {d} {rot} {layout} {dtype} {norm}")
    q, k, _, pos, freq, wq, wk = make(N, Hq, Hkv, d, rot, dtype, N + rot, norm, packed, gap=8 if packed else 0)
    scale = 1.2 if rot == 64 else 1.0
    qo, ko = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk, rot_scale=scale, layout=layout, out_f32=out_f32)
    torch.cuda.synchronize()
    for got, x, w, n in ((qo, q, wq, "q"), (ko, k, wk, "k")):
        assert got.dtype == (FL if out_f32 else dtype) and got.is_contiguous()
        assert_within(got, *ref(x, w, pos, freq, layout, scale=scale), got.dtype, n)


def test_positions():
    """Positions at and past the ends of the usual range; no frequency table
    without a rotated part; one side without a norm."""
    q, k, _, pos, freq, wq, _ = make(6, 4, 2, 128, 128, FL, 3)
    pos.copy_(torch.tensor([0, 1, -1, -2 ** 31, 2 ** 31 - 1, 10 ** 9], dtype=torch.int32))
    qo, ko = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, None)
    # the angle's own product is rounded twice in 64 bits: 2^31 radians to 2^-21
    slack = 2.0 ** -20
    for got, x, w in ((qo, q, wq), (ko, k, None)):
        y, b = ref(x, w, pos, freq, "half")
        assert_within(got, y, b + slack * b / (24 * F32), FL, "positions")
    qo, _ = hb.hybrid_qk_norm_rope(q, k, None, pos, wq, None)
    assert_within(qo, *ref(q, wq, pos, freq[:0], "half"), FL, "no rotation")


def test_no_tokens():
    q, k, _, pos, freq, wq, wk = make(0, 4, 2, 64, 64, BF, 1, packed=False)
    qo, ko = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    assert qo.shape == q.shape and ko.shape == k.shape
    dq, dk, dwq, dwk = hb.hybrid_qk_norm_rope_backward(q, k, q, k, freq, pos, wq, wk)
    torch.cuda.synchronize()
    assert dq.shape == q.shape and not dwq.any() and not dwk.any()


def test_outputs_in_one_buffer():
    """q_out and k_out as views of one packed buffer; the rest of it stays."""
    q, k, _, pos, freq, wq, wk = make(37, 4, 2, 64, 64, BF, 5)
    buf = torch.full((37, 8 * 64), 7.0, dtype=BF, device="cuda")
    qo, ko = buf[:, :256].unflatten(1, (4, 64)), buf[:, 256:384].unflatten(1, (2, 64))
    hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk, q_out=qo, k_out=ko)
    a, b = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    torch.cuda.synchronize()
    assert torch.equal(qo, a) and torch.equal(ko, b) and bool((buf[:, 384:] == 7.0).all())
    dq, dk, _, _ = hb.hybrid_qk_norm_rope_backward(q, k, a, b, freq, pos, wq, wk)
    hb.hybrid_qk_norm_rope_backward(q, k, a, b, freq, pos, wq, wk, dq=qo, dk=ko)
    torch.cuda.synchronize()
    assert torch.equal(qo, dq) and torch.equal(ko, dk) and bool((buf[:, 384:] == 7.0).all())


@pytest.mark.parametrize("N,Hq,Hkv,d,page,dtype,want_k", [
    (1, 16, 4, 128, 64, BF, True), (70, 12, 3, 64, 32, FL, False), (700, 8, 8, 128, 16, BF, False),
    (3000, 16, 4, 128, 64, BF, True)])
def test_paged(N, Hq, Hkv, d, page, dtype, want_k):
    announce(f"rope paged {N} {Hq} {Hkv} {d}")
    q, k, v, pos, freq, wq, wk = make(N, Hq, Hkv, d, d, dtype, N)
    n_pages = -(-N // page) + 3
    rows = n_pages * page
    g = torch.Generator().manual_seed(N)
    slots = torch.randperm(rows, generator=g)[:N].to(torch.int32)
    bad = [-1, -2 ** 31, rows, 2 ** 31 - 1]  # rows that are written nowhere
    for i, s in enumerate(bad[:N // 8]):
        slots[i * 7] = s
    kp = torch.randn(n_pages, page, Hkv, d, generator=g).to(dtype).cuda()
    vp = torch.randn(n_pages, page, Hkv, d, generator=g).to(dtype).cuda()
    kp0, vp0 = kp.clone(), vp.clone()
    slots = slots.cuda()
    qo, ko = hb.hybrid_qk_norm_rope_paged(q, k, v, freq, pos, slots, kp, vp, wq, wk, want_k=want_k)
    qr, kr = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    torch.cuda.synchronize()
    live = (slots >= 0) & (slots < rows)
    kp0.view(rows, Hkv, d)[slots[live].long()] = kr[live]
    vp0.view(rows, Hkv, d)[slots[live].long()] = v[live]
    assert torch.equal(qo, qr) and torch.equal(kp, kp0) and torch.equal(vp, vp0)
    assert (ko is None) == (not want_k) and (ko is None or torch.equal(ko, kr))


@pytest.mark.parametrize("N,Hq,Hkv,d,rot,layout,dtype,norm,packed", SHAPES)
@pytest.mark.parametrize("grad", [FL, BF])
def test_gradient(N, Hq, Hkv, d, rot, layout, dtype, norm, packed, grad):
    announce(f"rope backward {N} {Hq} {Hkv} {d} {rot} {layout} {dtype} {norm} {grad}")
    q, k, _, pos, freq, wq, wk = make(N, Hq, Hkv, d, rot, dtype, N + rot, norm, packed)
    g = torch.Generator().manual_seed(N + 9)
    up = [(0.1 * torch.randn(N, h, d, generator=g)).to(grad).cuda() for h in (Hq, Hkv)]
    scale = 1.2 if rot == 64 else 1.0
    call = lambda: hb.hybrid_qk_norm_rope_backward(q, k, *up, freq, pos, wq, wk, rot_scale=scale, layout=layout)
    got, again = call(), call()
    torch.cuda.synchronize()
    for x, w, u, dx, dw in ((q, wq, up[0], got[0], got[2]), (k, wk, up[1], got[1], got[3])):
        rx, rw, ex, ew = norm_rope_gradient(rows64(x), None if w is None else rows64(w), rows64(u),
                                            pos.cpu().numpy(), rows64(freq), layout, 1e-6, scale)
        assert dx.dtype == dtype
        assert_within(dx, rx, ex, dtype, "dx")
        assert (dw is None) == (w is None)
        if w is not None:
            assert_within(dw, rw, ew, FL, "dw")
    for a, b in zip(got, again):  # the same bits every time
        assert a is None or torch.equal(a, b)


def test_gradient_against_differences():
    """The fp32 gradient along random directions against central differences
    of the 64-bit forward."""
    q, k, _, pos, freq, wq, wk = make(9, 4, 2, 64, 32, FL, 11, packed=False)
    g = torch.Generator().manual_seed(1)
    up = [torch.randn(x.shape, generator=g).cuda() for x in (q, k)]
    dq, dk, dwq, dwk = hb.hybrid_qk_norm_rope_backward(q, k, *up, freq, pos, wq, wk)
    p, f = pos.cpu().numpy(), rows64(freq)
    rng = np.random.default_rng(2)

    def value(x, w, u):
        return float((norm_rope(x, w, p, f, "half", 1e-6, 1.0)[0] * u).sum())

    for x, w, u, dx, dw in ((q, wq, up[0], dq, dwq), (k, wk, up[1], dk, dwk)):
        x, w, u = rows64(x), rows64(w), rows64(u)
        tx, tw = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        h = 1e-5
        want = (value(x + h * tx, w + h * tw, u) - value(x - h * tx, w - h * tw, u)) / (2 * h)
        have = float((rows64(dx) * tx).sum() + (rows64(dw) * tw).sum())
        size = float(np.abs(rows64(dx) * tx).sum() + np.abs(rows64(dw) * tw).sum())
        # the differences' own error: h^2 times third derivatives, 1e-10 here, and 1e-16 / h
        assert abs(want - have) <= size * (200 * F32 + 1e-8), (want, have)


def test_zero_rows():
    """Rows of zeros: zero forward (eps keeps them finite), and a finite gradient."""
    q, k, _, pos, freq, wq, wk = make(4, 2, 1, 64, 64, FL, 7, packed=False)
    q.zero_()
    qo, _ = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    up = torch.ones_like(q), torch.ones_like(k)
    dq, _, dwq, _ = hb.hybrid_qk_norm_rope_backward(q, k, *up, freq, pos, wq, wk)
    rx, rw, ex, ew = norm_rope_gradient(rows64(q), rows64(wq), rows64(up[0]), pos.cpu().numpy(), rows64(freq), "half",
                                        1e-6, 1.0)
    assert not qo.any()
    assert_within(dq, rx, ex, FL, "dq at zero")
    assert_within(dwq, rw, ew, FL, "dwq at zero")


def test_other_stream_and_graph():
    """The same bits on a side stream, and from every replay of a captured call
    on new inputs and positions."""
    q, k, v, pos, freq, wq, wk = make(300, 8, 2, 128, 128, BF, 21)
    want = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk, stream=s)
    gb = hb.hybrid_qk_norm_rope_backward(q, k, *want, freq, pos, wq, wk, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    wb = hb.hybrid_qk_norm_rope_backward(q, k, *want, freq, pos, wq, wk)
    assert all(torch.equal(a, b) for a, b in zip(gb, wb))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
        back = hb.hybrid_qk_norm_rope_backward(q, k, *out, freq, pos, wq, wk)
    for i in range(3):
        q.copy_(torch.randn_like(q.float()).to(BF))
        pos.add_(17)
        graph.replay()
        torch.cuda.synchronize()
        o = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
        b = hb.hybrid_qk_norm_rope_backward(q, k, *o, freq, pos, wq, wk)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out + back, o + b)), i


def test_ways_to_call():
    """By name, and on a stream given as an object, a raw handle or the null stream."""
    q, k, _, pos, freq, wq, wk = make(70, 8, 2, 64, 64, BF, 3, packed=False)
    want = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream, 0, torch.cuda.default_stream()):
        got = hb.hybrid_qk_norm_rope(q=q, k=k, inv_freq=freq, positions=pos, wq=wq, wk=wk, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), stream
    with pytest.raises(ValueError):
        hb.hybrid_qk_norm_rope(q[:1].expand(70, 8, 64), k, freq, pos, wq, wk)
    with pytest.raises((TypeError, ValueError)):
        hb.hybrid_qk_norm_rope(q, k, freq.float(), pos, wq, wk)
    with pytest.raises((TypeError, ValueError)):
        hb.hybrid_qk_norm_rope(q, k, freq, pos.long(), wq, wk)
