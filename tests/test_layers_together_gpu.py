"""The operators around the softmax layers as they are used together: a
serving loop (page plan, norm and rotation into the pages, windowed step) and a
training step (norm and rotation, windowed prefill, and both gradients),
against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import F32, attend, norm_rope, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,window,sinks", [
    (FL, 8, 2, 64, 1, 20, 3), (BF, 16, 4, 128, 1, 40, 4), (BF, 8, 2, 128, 32, 64, 0), (FL, 4, 4, 64, 7, 31, 5)])
def test_serving(dtype, Hq, Hkv, d, L, window, sinks):
    """Three requests: prompts into the pages, then blocks of L tokens, one
    request at a time idle; every block's outputs are those of the whole sequence."""
    announce(f"serving {dtype} {Hq} {Hkv} {d} {L}")
    page, max_pages, B = 32, 8, 3
    g = torch.Generator().manual_seed(L + d)
    total = [L * n for n in (3, 5, 4)]
    prompt = [66, 31, 0]
    n_tok = [p + t for p, t in zip(prompt, total)]
    # projections of every token of every request
    x = [(1.3 * torch.randn(n, (Hq + 2 * Hkv) * d, generator=g)).to(dtype) for n in n_tok]
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2)]
    freq = (1e4 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).cuda()
    n_pages = 40
    kp = torch.full((n_pages, page, Hkv, d), float("nan"), dtype=dtype, device="cuda")
    vp = kp.clone()
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    held = [0] * B
    outs = [[] for _ in range(B)]

    def cached(new, sizes, max_tokens):
        """Plans `sizes` tokens per request, writes their keys and values; returns q, k, v rows."""
        nonlocal free
        lens = torch.tensor(held, dtype=torch.int32).cuda()
        slots, pos, start, counts = hb.kv_pages_plan(lens, torch.tensor(sizes, dtype=torch.int32).cuda(), table, free,
                                                     page, max_tokens)
        taken, missing = counts.tolist()
        assert missing == 0
        free = free[taken:].contiguous()
        packed = torch.zeros(max_tokens, (Hq + 2 * Hkv) * d, dtype=dtype)
        rows = torch.cat(new) if new else packed[:0]
        packed[:len(rows)] = rows
        packed = packed.cuda()
        q, k, v = (packed[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in
                   ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        q, k = hb.hybrid_qk_norm_rope_paged(q, k, v, freq, pos, slots, kp, vp, *w, want_k=True)
        return q, k, v, start.tolist(), lens

    cached([x[b][:prompt[b]] for b in range(B)], prompt, sum(prompt) + 5)
    held = list(prompt)
    for step in range(5):
        sizes = [L if len(outs[b]) * L < total[b] and (step + b) % 5 != 4 else 0 for b in range(B)]
        new = [x[b][held[b]:held[b] + sizes[b]] for b in range(B)]
        q, k, v, start, lens = cached(new, sizes, B * L + 3)
        blk = [torch.full((B, L, t.shape[1], d), float("nan"), dtype=dtype, device="cuda") for t in (q, k, v)]
        for b in range(B):
            for t, s in zip(blk, (q, k, v)):
                t[b, :sizes[b]] = s[start[b]:start[b] + sizes[b]]
        out = hb.softmax_window_step_paged(*blk, kp, vp, table, lens, window, sinks,
                                           block_len=torch.tensor(sizes, dtype=torch.int32).cuda(), out_f32=True)
        torch.cuda.synchronize()
        for b in range(B):
            if sizes[b]:
                outs[b].append((held[b], rows64(out[b])))
                held[b] += L
    for b in range(B):
        assert len(outs[b]) >= 2
        n = held[b]
        pos = np.arange(n)
        xr = rows64(x[b][:n])
        y = [norm_rope(xr[:, a * d:e * d].reshape(n, e - a, d), rows64(wt), pos, rows64(freq), "half", 1e-6, 1.0)[0]
             for (a, e), wt in (((0, Hq), w[0]), ((Hq, Hq + Hkv), w[1]))]
        vv = xr[:, (Hq + Hkv) * d:].reshape(n, Hkv, d)
        # q and k carry a rounding each (bf16: 2^-8 of a rotated entry), so a score
        # moves by up to 2^-7 of the sum of its terms' sizes
        eps = 2.0 ** -8 if dtype == BF else 32 * F32
        for at, got in outs[b]:
            for h in range(Hq):
                kk = y[1][:, h * Hkv // Hq]
                j = np.arange(at + L)
                j = j[(j < sinks) | (j >= at - window)]
                qq = y[0][at:at + L, h]
                o, _, err, _ = attend(qq, kk[j], vv[j, h * Hkv // Hq], np.ones((L, len(j)), bool), dtype == BF)
                move = 2 * eps * (np.abs(qq) @ np.abs(kk[j]).T).max(1, keepdims=True) / np.sqrt(d)
                sc = qq @ kk[j].T / np.sqrt(d)
                p = np.exp(sc - sc.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                bound = err + (2 * np.expm1(2 * move) + eps) * (p @ np.abs(vv[j, h * Hkv // Hq])) + eps * np.abs(o)
                assert (np.abs(got[:, h] - o) <= bound + 1e-6).all(), (b, at, h, np.abs(got[:, h] - o).max())


def test_training_step():
    """fp32: the loss's gradient through the whole chain, against autograd of
    the same chain in 64 bits, and the same bits from a captured chain."""
    B, T, Hq, Hkv, d, L, window, sinks = 2, 77, 6, 2, 64, 8, 24, 3
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn(B * T, (Hq + 2 * Hkv) * d, generator=g).cuda()
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in range(2))
    up = torch.randn(B, T, Hq, d, generator=g).cuda()
    freq = (1e4 ** (-torch.arange(16, dtype=torch.float64) / 16)).cuda()
    pos = torch.arange(T, dtype=torch.int32).repeat(B).cuda()

    def chain():
        q, k, v = qkv.split([Hq * d, Hkv * d, Hkv * d], 1)
        q, k = q.unflatten(1, (Hq, d)), k.unflatten(1, (Hkv, d))
        vv = v.contiguous().view(B, T, Hkv, d)
        qo, ko = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
        qo, ko = qo.view(B, T, Hq, d), ko.view(B, T, Hkv, d)
        out, lse = hb.softmax_window_prefill(qo, ko, vv, L, window, sinks)
        dq, dk, dv = hb.softmax_window_backward(qo, ko, vv, out, lse, up, L, window, sinks)
        # the gradient of the packed projection, written in place
        grad = torch.empty_like(qkv)
        gq, gk = grad[:, :Hq * d].unflatten(1, (Hq, d)), grad[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
        _, _, dwq, dwk = hb.hybrid_qk_norm_rope_backward(q, k, dq.view(B * T, Hq, d), dk.view(B * T, Hkv, d), freq, pos,
                                                         wq, wk, dq=gq, dk=gk)
        grad[:, (Hq + Hkv) * d:] = dv.view(B * T, Hkv * d)
        return out, grad, dwq, dwk

    got = chain()
    torch.cuda.synchronize()
    x, a, c = (t.double().cpu().requires_grad_() for t in (qkv, wq, wk))
    f, p = freq.cpu(), pos.cpu().double()

    def turn(y, w):
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w
        ang = p[:, None, None] * f
        e, o = y[..., :16], y[..., 16:32]
        return torch.cat([e * ang.cos() - o * ang.sin(), o * ang.cos() + e * ang.sin(), y[..., 32:]], -1)

    q, k, v = (t.reshape(B * T, -1, d) for t in x.split([Hq * d, Hkv * d, Hkv * d], 1))
    q, k, v = (t.view(B, T, -1, d).transpose(1, 2) for t in (turn(q, a), turn(k, c), v))
    k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
    mask = torch.from_numpy(seen_mask(T, L, window, sinks))
    w = torch.softmax((q @ k.transpose(-1, -2) / d ** 0.5).masked_fill(~mask, -float("inf")), -1)
    out = (w @ v).transpose(1, 2)
    (out * up.double().cpu()).sum().backward()
    # about a hundred fp32 roundings along the chain, of the size of the largest entries
    for t, r, n in zip(got, (out.detach(), x.grad, a.grad, c.grad), ("out", "grad", "dwq", "dwk")):
        err, size = float((t.double().cpu() - r).abs().max()), float(r.abs().max())
        assert err <= 400 * F32 * size, (n, err, size)
    chain()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = chain()
    for i in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = chain()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(captured, want)), i


def test_two_streams_at_once():
    """Two requests' calls on two streams, each with buffers of its own, at
    the same time: the bits of one after the other."""
    g = torch.Generator().manual_seed(1)
    ins = [[torch.randn(1, 600, h, 128, generator=g).to(BF).cuda() for h in (8, 2, 2, 8)] for _ in range(2)]

    def run(t):
        o, e = hb.softmax_window_prefill(*t[:3], 32, 200, 4)
        return (o, e) + hb.softmax_window_backward(*t[:3], o, e, t[3], 32, 200, 4)

    want = [run(t) for t in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = []
    for t, s in zip(ins, streams):
        with torch.cuda.stream(s):
            got.append([run(t) for _ in range(4)])
    torch.cuda.synchronize()
    for runs, w in zip(got, want):
        assert all(torch.equal(a, b) for r in runs for a, b in zip(r, w))
