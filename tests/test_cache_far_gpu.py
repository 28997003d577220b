"""The 8-bit cache and packed softmax where offsets pass 32 bits, and numbers past the
library's integers."""
import numpy as np
import torch
import pytest

from paper_2608_06628_amd import binding as hb

import _cache_ref as ref
from _helpers import announce
from _window_ref import assert_within, attend, gradient, rows64, seen_mask

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32).cuda()


def rnd(*shape):
    return torch.empty(shape, dtype=BF, device="cuda").normal_()


def test_pages():
    """The last pages of pools of more than 2^32 codes."""
    page, sb, Hkv, Hq, d, n = 64, 32, 8, 16, 128, 66000
    assert n * page * Hkv * d > 2 ** 32
    announce(f"8-bit pools of {n} pages of {page} x {Hkv} heads")
    torch.manual_seed(2)
    kp, vp = (torch.zeros(n, page, Hkv, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.zeros(n, page // sb, Hkv, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
              for _ in range(2))
    ids = [[n - 1, 3, n - 2], [1, n - 3, 0]]
    small = {p: i for i, p in enumerate(sorted(sum(ids, [])))}  # the pages' places in a small copy
    table, tab = torch.tensor(ids, dtype=torch.int32, device="cuda"), np.array([[small[p] for p in r] for r in ids])
    host = {x: (np.zeros((6, page, Hkv, d), np.uint8), np.zeros((6, page // sb, Hkv), np.uint8)) for x in "kv"}
    held = np.zeros(2, int)
    for new in ([150, 100], [5, 17]):
        at = np.concatenate([[0], np.cumsum(new)])
        k, v = rnd(at[-1], Hkv, d), 3 * rnd(at[-1], Hkv, d)
        hb.kv_pages_q8_write(k, v, kp, vp, ks, vs, table, i32(held), i32(at))
        for x, t in (("k", k), ("v", v)):
            ref.write(*host[x], rows64(t), tab, held, at)
        held += new
    pages = torch.tensor(sorted(small), device="cuda")
    for x, p, s in (("k", kp, ks), ("v", vp, vs)):
        assert np.array_equal(p.view(torch.uint8)[pages].cpu().numpy(), host[x][0])
        assert np.array_equal(s.view(torch.uint8)[pages].cpu().numpy(), host[x][1])
    at = np.concatenate([[0], np.cumsum(held)])
    k, v = hb.kv_pages_q8_read(kp, vp, ks, vs, table, i32([0, 0]), i32(at), tokens=int(at[-1]))
    cached = {x: [ref.values(*host[x])[tab[b, np.arange(m) // page], np.arange(m) % page] for b, m in enumerate(held)]
              for x in "kv"}
    for x, t in (("k", k), ("v", v)):
        assert np.array_equal(rows64(t), np.concatenate(cached[x]))
    for L in (1, 8, 32):
        q, k, v = rnd(2, L, Hq, d), rnd(2, L, Hkv, d), rnd(2, L, Hkv, d)
        for window, sinks in ((70, 5), (2 ** 40, 2 ** 33)):  # (the second see everything)
            out = hb.softmax_window_step_paged_q8(q, k, v, kp, vp, ks, vs, table, i32(held), window, sinks)
            torch.cuda.synchronize()
            for b, m in enumerate(held):
                j = np.array([x for x in range(m) if x >= m - window or x < sinks])
                kb, vb = (np.concatenate([cached[x][b][j], rows64(t[b])]) for x, t in (("k", k), ("v", v)))
                for h in range(Hq):
                    o, _, err, _ = attend(rows64(q[b, :, h]), kb[:, h // 2], vb[:, h // 2], np.ones((L, len(kb)), bool), True)
                    assert_within(out[b, :, h], o, err, BF, f"L={L} b={b} h={h}")


def test_rows():
    """Rows of more than 2^31 elements, into and out of the cache."""
    N, Hkv, d, page = 270000, 64, 128, 64
    assert N * Hkv * d > 2 ** 31
    announce(f"8-bit write and read of {N} x {Hkv} heads")
    torch.manual_seed(4)
    k, v = rnd(N, Hkv, d), rnd(N, Hkv, d)
    lens = [N - 100, 100]
    per = -(-lens[0] // page)
    n = per + 2
    table = torch.zeros(2, per, dtype=torch.int32)
    table[0], table[1, :2] = torch.arange(per), torch.tensor([per, per + 1])
    table = table.cuda()
    kp, vp = (torch.zeros(n, page, Hkv, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.zeros(n, 1, Hkv, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2))
    first, start = i32([0, 0]), i32([0, lens[0], N])
    hb.kv_pages_q8_write(k, v, kp, vp, ks, vs, table, first, start)
    bk, bv = hb.kv_pages_q8_read(kp, vp, ks, vs, table, first, start, tokens=N)
    torch.cuda.synchronize()
    last = lens[0] // page * page  # the first request's last page, and the second's
    for x, back in ((k, bk), (v, bv)):
        host = np.zeros((3, page, Hkv, d), np.uint8), np.zeros((3, 1, Hkv), np.uint8)
        ref.write(*host, rows64(x[last:]), np.array([[0, 0], [1, 2]]), np.zeros(2, int),
                  np.array([0, lens[0] - last, N - last]))
        val = ref.values(*host)
        want = np.concatenate([val[0, :lens[0] - last], val[1:].reshape(-1, Hkv, d)[:100]])
        assert np.array_equal(rows64(back[last:]), want)
        # (an entry is off by at most half a step: 2^-4 of it, or half of the least subnormal's
        # step times the scale, which is at most 2^-8 of the block's largest)
        for a in range(0, N, 30000):
            y = x[a:a + 30000].float()
            assert bool(((back[a:a + 30000].float() - y).abs() <= 2.0 ** -4 * y.abs() + 8 * 2.0 ** -17).all()), a


def test_packed_rows():
    """Sequences behind more than 2^31 elements, as views of one projection."""
    lens, Hq, Hkv, d, window = [200000, 69900, 100], 64, 1, 128, 48
    N = sum(lens)
    assert N * Hq * d > 2 ** 31
    announce(f"packed softmax of {N} x {Hq} heads")
    torch.manual_seed(3)
    x = rnd(N, (Hq + 2 * Hkv) * d)
    q, k, v = (x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, Hq), (Hq, Hq + 1), (Hq + 1, Hq + 2)))
    dout, start = rnd(N, Hq, d), i32([0, lens[0], lens[0] + lens[1], N])
    out, lse = hb.softmax_packed_prefill(q, k, v, start, 1, window)
    dq, dk, dv = hb.softmax_packed_backward(q, k, v, start, out, lse, dout, 1, window)
    torch.cuda.synchronize()
    # the last sequence, and the last rows of the one before (queries of its last 40 see no
    # key before them, and no query before them their keys)
    for a, b, n in ((N - 100, N, 100), (N - 100 - 96, N - 100, 40)):
        mask = seen_mask(b - a, 1, window, 0)
        sums = [0.0] * 4
        t = slice(b - n, b)
        for h in range(Hq):
            y = rows64(q[a:b, h]), rows64(k[a:b, 0]), rows64(v[a:b, 0])
            o, e, oerr, eerr = attend(*y, mask, True)
            assert_within(out[t, h], o[-n:], oerr[-n:], BF, f"out h={h}")
            assert_within(lse[h, t], e[-n:], eerr[-n:], FL, f"lse h={h}")
            r, g = gradient(*y, rows64(out[a:b, h]), rows64(lse[h, a:b]), rows64(dout[a:b, h]), mask, True)
            assert_within(dq[t, h], r[0][-n:], g[0][-n:], BF, f"dq h={h}")
            for i, s in enumerate((r[1], g[1], r[2], g[2])):
                sums[i] = sums[i] + s
        assert_within(dk[t, 0], sums[0][-n:], sums[1][-n:], BF, "dk")
        assert_within(dv[t, 0], sums[2][-n:], sums[3][-n:], BF, "dv")
    # a window and sinks past the library's integers see everything
    s = i32([0, 100])
    few = [m[-100:] for m in (q, k, v)]
    assert all(torch.equal(a, b) for a, b in zip(hb.softmax_packed_prefill(*few, s, 1, 2 ** 40, 2 ** 33),
                                                 hb.softmax_packed_prefill(*few, s, 1, 2 ** 31 - 1)))
