"""The 8-bit cache and packed sequences as they are used together: a serving loop (page
plan, norm and rotation, packed prompts, the cache's write, attention over it, its rows
handed to a recurrent state) and a training step (norm and rotation, packed softmax, and
both gradients)."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

import _cache_ref as ref
from _helpers import announce
from _window_ref import F32, assert_within, attend, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32
ALL = 2 ** 31 - 1


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,page,sb,window,sinks", [
    (BF, 16, 4, 128, 32, 64, 32, ALL, 0), (BF, 8, 2, 64, 1, 32, 32, 40, 4), (BF, 12, 4, 128, 7, 64, 64, 50, 3),
    (FL, 4, 2, 64, 8, 64, 32, ALL, 0)])
def test_serving(dtype, Hq, Hkv, d, L, page, sb, window, sinks):
    """Three prompts at once, then blocks of L tokens, one request at a time idle.  The
    cache holds exactly what its definition makes of the rotated keys, every block's
    outputs are those over the values it holds, and a state that takes the cached rows
    over is the one of those values."""
    announce(f"serving q8 {dtype} {Hq} {Hkv} {d} {L}")
    B, max_pages, n_pages = 3, 8, 30
    g = torch.Generator().manual_seed(L + d)
    prompt = [66, 1, 130]
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2)]
    freq = (1e4 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).cuda()
    cache = ref.Cache(n_pages, page, sb, Hkv, d, L)
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    held = [0] * B

    def new_rows(sizes, behind):
        """Plans `sizes` tokens per request; their rotated q, k and their v, with `behind` rows of padding."""
        nonlocal free
        lens, n = i32(held), sum(sizes) + behind
        _, pos, start, counts = hb.kv_pages_plan(lens, i32(sizes), table, free, page, n)
        taken, missing = counts.tolist()
        assert missing == 0
        free = free[taken:].contiguous()
        x = torch.randn(n, (Hq + 2 * Hkv) * d, generator=g).to(dtype).cuda()
        q, k, v = (x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in
                   ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        q, k = hb.hybrid_qk_norm_rope(q, k, freq, pos, *w)
        return q, k, v, start, lens

    def store(k, v, lens, start, sizes):
        before = [cache.codes(x) for x in "kv"]
        hb.kv_pages_q8_write(k, v, *cache.args, table, lens, start)
        at = np.concatenate([[0], np.cumsum(sizes)])
        for i, (x, t) in enumerate((("k", k), ("v", v))):
            cache.host[x] = tuple(a.copy() for a in before[i])
            ref.write(*cache.host[x], rows64(t), table.cpu().numpy(), np.array(held), at)
            for a, b in zip(cache.codes(x), cache.host[x]):
                assert np.array_equal(a, b), x
        for b in range(B):
            held[b] += sizes[b]

    def value(x, b):
        """Request b's cached values."""
        p = np.arange(held[b])
        return ref.values(*cache.host[x])[table.cpu().numpy()[b, p // page], p % page]

    q, k, v, start, lens = new_rows(prompt, 5)
    out, lse = hb.softmax_packed_prefill(q, k, v, start, L, window, sinks)
    at = start.tolist()
    assert at == np.concatenate([[0], np.cumsum(prompt)]).tolist()
    for a, b in zip(at, at[1:]):
        for h in range(Hq):
            o, e, oerr, eerr = attend(rows64(q[a:b, h]), rows64(k[a:b, h * Hkv // Hq]), rows64(v[a:b, h * Hkv // Hq]),
                                      seen_mask(b - a, L, window, sinks), dtype == BF)
            assert_within(out[a:b, h], o, oerr, dtype, f"prompt {a} {h}")
            assert_within(lse[h, a:b], e, eerr, FL, f"prompt lse {a} {h}")
    store(k, v, lens, start, prompt)
    for step in range(4):
        sizes = [0 if (step + b) % 4 == 3 else L for b in range(B)]
        q, k, v, start, lens = new_rows(sizes, 3)
        at = start.tolist()
        blk = [torch.full((B, L, t.shape[1], d), float("nan"), dtype=dtype, device="cuda") for t in (q, k, v)]
        for b in range(B):
            for t, s in zip(blk, (q, k, v)):
                t[b, :sizes[b]] = s[at[b]:at[b + 1]]
        out = hb.softmax_window_step_paged_q8(*blk, *cache.args, table, lens, window, sinks, block_len=i32(sizes))
        torch.cuda.synchronize()
        for b in range(B):
            assert sizes[b] or not out[b].any()
            for h in range(Hq if sizes[b] else 0):
                j = np.arange(held[b])
                j = j[(j < sinks) | (j >= held[b] - window)]
                kk, vv = (np.concatenate([value(x, b)[j, h * Hkv // Hq], rows64(t[b, :, h * Hkv // Hq])])
                          for x, t in (("k", blk[1]), ("v", blk[2])))
                o, _, err, _ = attend(rows64(blk[0][b, :, h]), kk, vv, np.ones((L, len(kk)), bool), dtype == BF)
                assert_within(out[b, :, h], o, err, dtype, f"step {step} {b} {h}")
        store(k, v, lens, start, sizes)
    # the cached tokens of two requests as rows, behind a first part that stays where it is
    skip = [held[0] - 32, 0, held[2] - 64]
    n = [held[b] - skip[b] for b in range(B)]
    n[1] = 0
    start = i32(np.concatenate([[0], np.cumsum(n)]))
    k, v = hb.kv_pages_q8_read(*cache.args, table, i32(skip), start, tokens=sum(n), dtype=dtype)
    torch.cuda.synchronize()
    for x, t in (("k", k), ("v", v)):
        assert np.array_equal(rows64(t), np.concatenate([value(x, b)[skip[b]:skip[b] + n[b]] for b in (0, 2)]))
    W = (torch.randn(Hq, 64, d, generator=g) / d ** 0.5).to(dtype).cuda()
    S, z = torch.zeros(3, Hq, d, 128, device="cuda"), torch.zeros(3, Hq, 128, device="cuda")
    kb, vb = k.view(3, 32, Hkv, d), v.view(3, 32, Hkv, d)
    want = S.clone(), z.clone()
    hb.hybrid_state_commit(kb, vb, W, S, z)
    host = [torch.from_numpy(np.concatenate([value(x, b)[skip[b]:] for b in (0, 2)])).to(dtype).cuda().view(3, 32, Hkv, d)
            for x in "kv"]
    hb.hybrid_state_commit(*host, W, *want)
    torch.cuda.synchronize()
    assert bool(S.any()) and torch.equal(S, want[0]) and torch.equal(z, want[1])


def test_training_step():
    """fp32: the loss's gradient through the whole chain of a packed batch, against
    autograd of the same chain in 64 bits a sequence at a time, and the same bits from a captured chain."""
    announce("packed training step")
    lens, Hq, Hkv, d, L, window, sinks, tail = [77, 1, 40], 6, 2, 64, 8, 24, 3, 4
    g = torch.Generator().manual_seed(5)
    at = np.concatenate([[0], np.cumsum(lens)]).tolist()
    n = at[-1]
    qkv = torch.randn(n + tail, (Hq + 2 * Hkv) * d, generator=g).cuda()
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in range(2))
    up = torch.randn(n + tail, Hq, d, generator=g).cuda()
    freq = (1e4 ** (-torch.arange(16, dtype=torch.float64) / 16)).cuda()
    pos = torch.cat([torch.arange(m, dtype=torch.int32) for m in lens + [tail]]).cuda()
    start = i32(at)

    def chain():
        q, k, v = qkv.split([Hq * d, Hkv * d, Hkv * d], 1)
        q, k, v = q.unflatten(1, (Hq, d)), k.unflatten(1, (Hkv, d)), v.unflatten(1, (Hkv, d))
        qo, ko = hb.hybrid_qk_norm_rope(q, k, freq, pos, wq, wk)
        out, lse = hb.softmax_packed_prefill(qo, ko, v, start, L, window, sinks)
        dq, dk, dv = hb.softmax_packed_backward(qo, ko, v, start, out, lse, up, L, window, sinks)
        grad = torch.empty_like(qkv)  # of the packed projection, written in place
        gq, gk = grad[:, :Hq * d].unflatten(1, (Hq, d)), grad[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
        _, _, dwq, dwk = hb.hybrid_qk_norm_rope_backward(q, k, dq, dk, freq, pos, wq, wk, dq=gq, dk=gk)
        grad[:, (Hq + Hkv) * d:] = dv.flatten(1)
        return out, grad, dwq, dwk

    got = chain()
    torch.cuda.synchronize()
    assert not got[0][n:].any() and not got[1][n:].any()
    x, a, c = (t.double().cpu().requires_grad_() for t in (qkv, wq, wk))
    f = freq.cpu()

    def turn(y, w):
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w
        ang = torch.arange(len(y), dtype=torch.float64)[:, None, None] * f
        e, o = y[..., :16], y[..., 16:32]
        return torch.cat([e * ang.cos() - o * ang.sin(), o * ang.cos() + e * ang.sin(), y[..., 32:]], -1)

    outs = []
    for s, e in zip(at, at[1:]):
        q, k, v = (t.reshape(e - s, -1, d) for t in x[s:e].split([Hq * d, Hkv * d, Hkv * d], 1))
        q, k, v = (t.transpose(0, 1) for t in (turn(q, a), turn(k, c), v))
        k, v = (t.repeat_interleave(Hq // Hkv, 0) for t in (k, v))
        mask = torch.from_numpy(seen_mask(e - s, L, window, sinks))
        w = torch.softmax((q @ k.transpose(-1, -2) / d ** 0.5).masked_fill(~mask, -float("inf")), -1)
        outs.append((w @ v).transpose(0, 1))
    out = torch.cat(outs)
    (out * up[:n].double().cpu()).sum().backward()
    # about a hundred fp32 roundings along the chain, of the size of the largest entries
    for t, r, name in zip((got[0][:n], got[1][:n]) + got[2:], (out.detach(), x.grad[:n], a.grad, c.grad),
                          ("out", "grad", "dwq", "dwk")):
        err, size = float((t.double().cpu() - r).abs().max()), float(r.abs().max())
        assert err <= 400 * F32 * size, (name, err, size)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = chain()
    for i, now in enumerate((at, [0, 40, 40, n], [0, 0, 100, 101])):
        start.copy_(i32(now))
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = chain()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(captured, want)), i


def test_two_streams_at_once():
    """Two servers' caches on two streams at the same time, each with buffers of its
    own, and two packed gradients: the bits of one after the other."""
    announce("q8 and packed on two streams")
    Hq, Hkv, d, L, B, page, sb = 16, 4, 128, 32, 4, 64, 32
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()
    table = torch.randperm(B * 20, generator=g).to(torch.int32).view(B, 20).cuda()
    lens, start = [1200, 31, 700, 64], i32(np.concatenate([[0], np.cumsum([1200, 31, 700, 64])]))
    n = sum(lens)
    ins = [(rnd(n, Hkv, d), rnd(n, Hkv, d), rnd(B, L, Hq, d), rnd(B, L, Hkv, d), rnd(B, L, Hkv, d), rnd(n, Hq, d),
            rnd(n, Hq, d)) for _ in range(2)]
    first, held = i32([0] * B), i32(lens)

    caches = [ref.Cache(B * 20, page, sb, Hkv, d, 3) for _ in range(8)]

    def run(t, c, stream=None):
        hb.kv_pages_q8_write(t[0], t[1], *c.args, table, first, start, stream=stream)
        o = hb.softmax_window_step_paged_q8(*t[2:5], *c.args, table, held, ALL, stream=stream)
        k, v = hb.kv_pages_q8_read(*c.args, table, first, start, tokens=n, stream=stream)
        out, lse = hb.softmax_packed_prefill(t[5], t[0], t[1], start, L, ALL, stream=stream)
        return (o, k, v, out, lse) + hb.softmax_packed_backward(t[5], t[0], t[1], start, out, lse, t[6], L, ALL,
                                                                stream=stream) + c.args

    want = [run(t, c) for t, c in zip(ins, caches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = [run(ins[i % 2], caches[2 + i], streams[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(r, want[i % 2])), i


def test_graphs_in_turn():
    """Two captured servers' steps, each with a workspace of its own, replayed in turn on
    changing lengths: the eager bits."""
    announce("q8 two graphs")
    Hq, Hkv, d, B, page, sb = 8, 2, 128, 2, 64, 64
    g = torch.Generator().manual_seed(2)
    sides = []
    for L in (1, 16):
        c = ref.Cache(80, page, sb, Hkv, d, L)
        for x in "kv":  # (any codes but NaN)
            c.host[x][0][...] &= 0xF7
        c.send()
        x = [torch.randn(B, L, h, d, generator=g).to(BF).cuda() for h in (Hq, Hkv, Hkv)]
        table = torch.randperm(80, generator=g).to(torch.int32).view(B, 40).cuda()
        lens, out = i32([2000, 700]), torch.zeros_like(x[0])
        call = lambda x=x, c=c, table=table, lens=lens, **kw: hb.softmax_window_step_paged_q8(
            *x, *c.args, table, lens, ALL, **kw)
        call(out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out=out)
        sides.append((graph, call, lens, out))
    for now in ([2000, 700], [0, 2560], [33, 1], [2559, 2559]):
        for graph, _, lens, out in sides:
            lens.copy_(i32(now))
            out.zero_()
        torch.cuda.synchronize()
        for graph, *_ in sides + sides[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for _, call, _, out in sides:
            assert torch.equal(out, call()), now
