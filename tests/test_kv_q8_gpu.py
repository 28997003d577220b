"""Writing an 8-bit cache and reading it back, against a host loop: equal, code by code."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

import _cache_ref as ref
from _helpers import announce

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def tables(B, per, n_pages, seed):
    return np.random.RandomState(seed).permutation(n_pages)[:B * per].reshape(B, per).astype(np.int32)


def rows(N, H, d, dtype, seed, scale=1.0):
    """k contiguous, v a view of wider rows, with channels of very different sizes."""
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(1.5 * torch.randn(H, d, generator=g)) * scale
    k = (torch.randn(N, H, d, generator=g) * size).to(dtype).cuda()
    v = (torch.randn(N, (H + 2) * d, generator=g) * scale).to(dtype).cuda()[:, 2 * d:].unflatten(1, (H, d))
    return k, v


def same(got, want, what):
    codes, scales = got
    nan = (codes & 127) == 127
    assert np.array_equal(nan, (want[0] & 127) == 127), f"{what}: NaNs elsewhere"
    assert np.array_equal(codes[~nan], want[0][~nan]), f"{what}: codes differ"
    assert np.array_equal(scales, want[1]), f"{what}: scales differ"


def write(cache, k, v, table, first, start, what):
    announce(what)
    hb.kv_pages_q8_write(k, v, *cache.args, i32(table), i32(first), i32(start))
    torch.cuda.synchronize()
    for x, t in (("k", k), ("v", v)):
        ref.write(*cache.host[x], t.double().cpu().numpy(), table, first, np.array(start, dtype=np.int64))
        same(cache.codes(x), cache.host[x], f"{what}: {x}")


SHAPES = [  # dtype, Hkv, d, page, sb
    (BF, 4, 128, 64, 32), (BF, 4, 128, 64, 64), (FL, 2, 64, 32, 32), (BF, 1, 64, 128, 128), (FL, 3, 128, 512, 256),
    (BF, 2, 128, 1024, 1024)]


@pytest.mark.parametrize("dtype,H,d,page,sb", SHAPES)
def test_write(dtype, H, d, page, sb):
    """Requests of no, one and many tokens, from a block's first row and from its middle,
    then the tokens that follow, larger by turns, so that blocks that go on grow."""
    new = [0, 1, 3 * sb + 5, sb, 2, page + 1, 31]
    held = [5, 0, 7, sb, page - 1, sb - 1, 0]
    B, per = len(new), -(-(max(new) + max(held) + 3 * sb) // page) + 1
    cache = ref.Cache(B * per + 2, page, sb, H, d, 1)
    table = tables(B, per, B * per + 2, 2)
    for step, scale in enumerate((1.0, 30.0, 0.01, 1000.0)):
        start = np.concatenate([[0], np.cumsum(new)])
        k, v = rows(int(start[-1]) + 3, H, d, dtype, 10 + step, scale)
        write(cache, k, v, table, held, start, f"write {dtype} {H} {d} {page} {sb} step {step}")
        held = [h + n for h, n in zip(held, new)]
        new = [1, 0, 2, sb // 2, 1, 1, sb + 1]


def test_write_special_values():
    """Zeros, infinities, NaN, the largest and the smallest numbers, exact powers of two
    and the edges of the scale's choice."""
    H, d, page, sb = 2, 64, 32, 32
    x = np.zeros((12 * sb, H, d), np.float32)
    x[1 * sb, 0, 0] = np.inf
    x[1 * sb + 1, 0, 1] = 3.0
    x[2 * sb, 0, 0], x[2 * sb, 1, 1] = np.nan, -np.inf
    x[3 * sb, 0, 0], x[3 * sb, 1, 0] = 3.4028235e38, -3.3895314e38
    x[4 * sb, 0, 0], x[4 * sb, 1, 0] = 1e-45, 2.0 ** -126
    x[5 * sb, 0, 0], x[5 * sb, 1, 0] = 448.0, np.nextafter(np.float32(448.0), np.float32(500.0))
    x[6 * sb:7 * sb] = (np.arange(sb * H * d).reshape(sb, H, d) - 2048) / 256.0  # every code, ties among them
    x[7 * sb:8 * sb, :, 0] = 447.0
    x[7 * sb:8 * sb, :, 1:] = 2.0 ** -np.arange(1, d)
    x[8 * sb] = 448.0 * 2.0 ** -117
    x[9 * sb] = -0.0
    x[10 * sb, 0, 0], x[10 * sb, 0, 1] = 448.0, 2.0 ** -10  # half the least code: a tie with zero
    x[11 * sb, 0, :3] = 448.0, 3 * 2.0 ** -10, 2.0 ** -10 * 1.0001
    cache = ref.Cache(12, page, sb, H, d, 3)
    t = torch.from_numpy(x).cuda()
    write(cache, t, t, tables(1, 12, 12, 4), [0], [0, len(x)], "write special values")
    k, v = hb.kv_pages_q8_read(*cache.args, i32(tables(1, 12, 12, 4)), i32([0]), i32([0, len(x)]), tokens=len(x), dtype=FL)
    got = k.cpu().numpy()
    assert np.isnan(got[1 * sb, 0, 0]) and got[1 * sb + 1, 0, 1] == 3.0  # an infinity leaves the others their scale
    assert torch.equal(torch.nan_to_num(k, 7.0), torch.nan_to_num(v, 7.0))


def test_growing_keeps_earlier_tokens():
    """A block written one token at a time, each larger than those before: the values of
    earlier tokens stay within half a step of e4m3 (2^-4 of a value, or half the least code
    times the scale), though they are rounded again and again."""
    announce("growing")
    H, d, page, sb = 1, 64, 32, 32
    cache = ref.Cache(1, page, sb, H, d, 5)
    x = (torch.randn(sb, H, d, generator=torch.Generator().manual_seed(6)) * 1.7 ** torch.arange(sb)[:, None, None]).cuda()
    for t in range(sb):
        write(cache, x[t:t + 1], x[t:t + 1], np.zeros((1, 1), np.int32), [t], [0, 1], f"growing {t}")
    k, _ = hb.kv_pages_q8_read(*cache.args, i32([[0]]), i32([0]), i32([0, sb]), tokens=sb, dtype=FL)
    step = 2.0 ** (float(cache.codes("k")[1][0, 0, 0]) - 127 - 9)
    # (once per growth below 2^-6 of the scale: their halves of ever larger steps sum to one step)
    assert bool(((k - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), torch.tensor(step).cuda()) + step).all())


def test_out_of_range():
    """Pages outside the pool, tokens past the page table and past the rows given, a
    negative first: nothing else is written, and reading leaves those rows as they were."""
    H, d, page, sb, n_pages = 2, 128, 32, 32, 9
    table = np.array([[0, -1, 1], [9, 2, 3], [4, 5, 2 ** 31 - 1], [6, 7, 8]], np.int32)
    new, held = [70, 50, 60, 40], [10, 20, -5, 90]
    start = np.concatenate([[0], np.cumsum(new)])
    k, v = rows(int(start[-1]) - 20, H, d, BF, 7)  # (fewer rows than token_start says)
    cache = ref.Cache(n_pages, page, sb, H, d, 8)
    write(cache, k, v, table, held, start, "out of range")
    k2, v2 = (torch.full_like(t.contiguous(), 5.0) for t in (k, v))
    hb.kv_pages_q8_read(*cache.args, i32(table), i32(held), i32(start), k=k2, v=v2)
    torch.cuda.synchronize()
    want = {x: np.full(tuple(k.shape), 5.0) for x in "kv"}
    for b in range(4):
        for i in range(new[b]):
            p, t = max(held[b], 0) + i, start[b] + i
            if t < len(k) and p < 96 and 0 <= table[b, p // page] < n_pages:
                for x in "kv":
                    want[x][t] = ref.values(*cache.host[x])[table[b, p // page], p % page]
    assert np.array_equal(k2.double().cpu().numpy(), want["k"]) and np.array_equal(v2.double().cpu().numpy(), want["v"])


@pytest.mark.parametrize("dtype,H,d,page,sb", SHAPES)
@pytest.mark.parametrize("B,most", [(1, 1), (3, 200), (70, 40), (300, 9)])
def test_read(dtype, H, d, page, sb, B, most):
    announce(f"read {dtype} {H} {d} {page} {sb} {B} {most}")
    r = np.random.RandomState(B + most)
    new, held = r.randint(0, most + 1, B), r.randint(0, 300, B)
    new[0] = most
    start = np.concatenate([[0], np.cumsum(new)])
    per = -(-(most + 300) // page)
    n_pages = max(8, min(B * per, 64))
    table = r.randint(0, n_pages, (B, per)).astype(np.int32)  # (pages may be shared)
    cache = ref.Cache(n_pages, page, sb, H, d, 9)
    for x in "kv":
        cache.host[x][0][(cache.host[x][0] & 127) == 127] = 1
    cache.send()
    N = int(start[-1]) + 4
    buf = torch.full((N, 2 * H * d + 8), 3.0, dtype=dtype, device="cuda")
    k, v = buf[:, :H * d].unflatten(1, (H, d)), buf[:, H * d + 8:].unflatten(1, (H, d))  # interleaved rows
    hb.kv_pages_q8_read(*cache.args, i32(table), i32(held), i32(start), k=k, v=v)
    torch.cuda.synchronize()
    for x, t in (("k", k), ("v", v)):
        full = ref.values(*cache.host[x])
        got = t.double().cpu().numpy()
        for b in range(B):
            p = held[b] + np.arange(new[b])
            assert np.array_equal(got[start[b]:start[b + 1]], full[table[b, p // page], p % page]), (x, b)
        assert (got[start[-1]:] == 3.0).all()
    assert bool((buf[:, H * d:H * d + 8] == 3.0).all())


def test_many_requests():
    """More requests than two looks at 64 starts find, most of them empty."""
    B, H, d, page, sb = 5000, 1, 64, 32, 32
    new = np.zeros(B, np.int64)
    new[[0, 63, 64, 65, 4095, 4096, 4097, 4999]] = [3, 40, 1, 33, 7, 64, 2, 5]
    start = np.concatenate([[0], np.cumsum(new)])
    held = np.arange(B) % 50
    cache = ref.Cache(40, page, sb, H, d, 11)
    table = np.full((B, 4), -1, np.int32)
    table[new > 0] = np.random.RandomState(12).permutation(40)[:32].reshape(8, 4)
    k, v = rows(int(start[-1]), H, d, BF, 13)
    write(cache, k, v, table, held, start, "many requests")


def test_captured():
    """A captured write plans from the lengths of each replay, and matches the eager one."""
    announce("captured write and read")
    H, d, page, sb, B = 4, 128, 64, 32, 3
    cache = ref.Cache(12, page, sb, H, d, 14)
    table = tables(B, 4, 12, 15)
    k, v = rows(64, H, d, BF, 16)
    tab, first, start = i32(table), i32([0, 0, 0]), i32([0, 0, 0, 0])
    k2, v2 = torch.zeros_like(k), torch.zeros_like(k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hb.kv_pages_q8_write(k, v, *cache.args, tab, first, start)
        hb.kv_pages_q8_read(*cache.args, tab, first, start, k=k2, v=v2)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hb.kv_pages_q8_write(k, v, *cache.args, tab, first, start)
        hb.kv_pages_q8_read(*cache.args, tab, first, start, k=k2, v=v2)
    torch.cuda.synchronize()
    for x in "kv":  # (the empty calls wrote nothing)
        same(cache.codes(x), cache.host[x], "before")
    held = np.zeros(B, np.int64)
    for n in ([5, 0, 40], [1, 1, 1], [30, 33, 0]):
        at = np.concatenate([[0], np.cumsum(n)])
        first.copy_(i32(held)), start.copy_(i32(at)), k.mul_(1.7)
        g.replay()
        torch.cuda.synchronize()
        for x, t, back in (("k", k, k2), ("v", v, v2)):
            ref.write(*cache.host[x], t.double().cpu().numpy(), table, held, at)
            same(cache.codes(x), cache.host[x], f"replay {n}")
            full = ref.values(*cache.host[x])
            for b in range(B):
                p = held[b] + np.arange(n[b])
                assert np.array_equal(back[at[b]:at[b + 1]].double().cpu().numpy(), full[table[b, p // page], p % page])
        held += n
