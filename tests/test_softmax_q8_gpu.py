"""softmax_window_step_paged_q8 against 64 bits on the values the cache holds: what of it
is seen, and that nothing else plays a part."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

import _cache_ref as ref
from _helpers import announce
from _window_ref import assert_within, attend, rows64

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32
ALL = 2 ** 31 - 1


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32).cuda()


def seen(n, window, sinks):
    j = np.arange(n)
    return j[(j >= n - window) | (j < sinks)]


def make(B, L, Hq, Hkv, d, page, sb, lens, dtype, seed, window, sinks):
    """Every cached row that is not seen, and every scale of no row that is, is NaN; entries
    of the table that are not read name pages far outside the pool."""
    g = torch.Generator().manual_seed(seed)
    r = np.random.RandomState(seed)
    per = -(-max(list(lens) + [1]) // page) + 1
    n = B * per + 2
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    table = r.permutation(n)[:B * per].reshape(B, per)
    cache = ref.Cache(n, page, sb, Hkv, d, seed)
    keep = np.zeros((n, page), bool)
    read = np.zeros((B, per), bool)
    for b, m in enumerate(lens):
        j = seen(m, window, sinks)
        keep[table[b, j // page], j % page] = True
        read[b, j // page] = True
    for x in "kv":
        codes, scales = cache.host[x]
        # values of unit size, whose blocks' scales differ
        scales[:] = r.randint(118, 124, scales.shape)
        z = r.standard_normal(codes.shape) * 2.0 ** (127 - scales.astype(np.float64)).repeat(sb, 1)[..., None]
        codes[:] = ref.encode(np.clip(z, -448, 448))
        codes[~keep] = 127
        scales[~keep.reshape(n, page // sb, sb).any(2)] = 255
    cache.send()
    t = np.where(read, table, 2 ** 31 - 1).astype(np.int32)
    return dict(q=rnd(B, L, Hq, d), k=rnd(B, L, Hkv, d), v=rnd(B, L, Hkv, d), cache=cache, host=table,
                table=torch.from_numpy(t).cuda(), lens=list(lens), page=page, window=window, sinks=sinks)


def expect(c, b, m):
    """(out, bound) [m, Hq, d] of request b's first m queries."""
    Hq, Hkv = c["q"].shape[2], c["k"].shape[2]
    j = seen(c["lens"][b], c["window"], c["sinks"])
    at = c["host"][b, j // c["page"]], j % c["page"]
    kb, vb = (np.concatenate([ref.values(*c["cache"].host[x])[at], rows64(c[x][b, :m])]) for x in "kv")
    res = [attend(rows64(c["q"][b, :m, h]), kb[:, h * Hkv // Hq], vb[:, h * Hkv // Hq], np.ones((m, len(kb)), bool),
                  c["q"].dtype == BF) for h in range(Hq)]
    return np.stack([x[0] for x in res], 1), np.stack([x[2] for x in res], 1)


def run(c, block, **kw):
    return hb.softmax_window_step_paged_q8(c["q"], c["k"], c["v"], *c["cache"].args, c["table"], i32(c["lens"]),
                                           c["window"], c["sinks"], block_len=None if block is None else i32(block), **kw)


def check(c, block=None, what=""):
    B, L = c["q"].shape[:2]
    dtype = c["q"].dtype
    for f32 in ([False, True] if dtype == BF else [False]):
        out = torch.full_like(c["q"], 9.0, dtype=FL if f32 else dtype)
        run(c, block, out=out)
        torch.cuda.synchronize()
        for b in range(B):
            m = L if block is None else min(max(block[b], 0), L)
            assert bool((out[b, m:] == 9.0).all()), f"{what}: rows past the block were written"
            if m:
                assert_within(out[b, :m], *expect(c, b, m), out.dtype, f"{what} b={b}")


CASES = [  # B, L, Hq, Hkv, d, page, sb, lens, window, sinks, dtype
    (1, 1, 1, 1, 64, 32, 32, [0], 5, 3, BF),
    (1, 1, 4, 1, 128, 32, 32, [1], 0, 0, BF),
    (3, 1, 4, 1, 128, 64, 32, [31, 32, 33], ALL, 0, BF),
    (5, 1, 16, 4, 128, 64, 64, [4097, 64, 31, 0, 500], 200, 4, BF),
    (5, 1, 16, 4, 128, 64, 32, [4097, 64, 31, 0, 500], ALL, 0, BF),
    (4, 32, 16, 4, 128, 64, 64, [1000, 33, 640, 2048], 96, 32, BF),
    (4, 32, 16, 4, 128, 64, 32, [1000, 33, 640, 2048], 0, 0, BF),
    (4, 32, 16, 4, 128, 64, 32, [1000, 33, 640, 2048], 0, 5, BF),
    (4, 32, 16, 4, 128, 64, 32, [1000, 33, 640, 2048], ALL, 0, BF),
    (2, 17, 8, 8, 64, 256, 256, [700, 3], 65, 1, BF),
    (2, 32, 8, 1, 64, 128, 64, [300, 257], 31, 100, BF),
    (2, 5, 12, 4, 128, 32, 32, [333, 97], 100, 7, BF),
    (2, 3, 10, 2, 64, 32, 32, [160, 95], ALL, 0, BF),
    (1, 32, 16, 1, 128, 64, 64, [500], 300, 40, BF),   # 16 query heads per KV head
    (2, 1, 48, 1, 64, 64, 32, [200, 31], ALL, 0, BF),   # 48
    (3, 32, 16, 4, 128, 64, 32, [0, 1, 32], ALL, 0, BF),  # a block alone, and two tiles
    (3, 32, 12, 2, 64, 32, 32, [0, 70, 650], 200, 3, BF),  # 6 tiles of columns
    (2, 29, 9, 3, 128, 32, 32, [95, 64], ALL, 0, BF),     # 3
    (1, 32, 4, 1, 128, 64, 64, [12000], ALL, 0, BF),
    (70, 1, 4, 2, 64, 64, 64, [(i * 37) % 200 for i in range(70)], ALL, 0, BF),
    (1, 1, 16, 4, 128, 64, 64, [20000], ALL, 0, BF),   # several ranges
    (2, 32, 4, 1, 64, 64, 64, [9000, 100], ALL, 0, BF),
    (3, 1, 8, 4, 64, 64, 32, [900, 0, 64], ALL, 0, FL),
    (2, 32, 16, 4, 128, 64, 64, [200, 75], 100, 5, FL),
    (1, 7, 3, 1, 128, 32, 32, [1000], ALL, 0, FL),
    (1, 1, 4, 2, 64, 32, 32, [6000], 5000, 33, FL)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:7]) + f"-{c[7][0]}-{c[8]}-{c[9]}-{str(c[10])[6:]}")
def test_step(case):
    announce(f"softmax q8 {case}")
    B, L, Hq, Hkv, d, page, sb, lens, window, sinks, dtype = case
    c = make(B, L, Hq, Hkv, d, page, sb, lens, dtype, L + d + len(lens), window, sinks)
    check(c, what="whole blocks")
    if L > 1:
        check(c, [[1, L, 0, L - 1, 2][b % 5] for b in range(B)], "active rows")


def test_no_cache_at_all():
    """max_pages = 0: the block alone."""
    announce("softmax q8 without pages")
    c = make(2, 8, 4, 2, 64, 32, 32, [0, 0], BF, 3, ALL, 0)
    c["table"] = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    check(c, what="no pages")


@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 1), (32, 32), (33, 31), (64, 33), (100, 64), (5, 200), (0, 64),
                                          (0, 31), (127, 0)])
@pytest.mark.parametrize("L", [1, 32])
def test_edges_of_the_window(window, sinks, L):
    announce(f"softmax q8 window {window} {sinks} {L}")
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 160, 257]
    check(make(len(lens), L, 4, 2, 64, 32, 32, lens, BF, window + sinks, window, sinks), what=f"{window} {sinks}")


def test_scores_that_climb_and_fall():
    """Keys whose scores rise or fall along the prefix by hundreds: the reference moves
    every tile, or never."""
    announce("softmax q8 climbing")
    for sign in (1.0, -1.0):
        c = make(1, 4, 4, 1, 64, 32, 32, [700], BF, 21, ALL, 0)
        codes, scales = c["cache"].host["k"]
        scales[:] = 127
        codes[:] = 0
        j = np.arange(700)
        codes[c["host"][0, j // 32], j % 32, 0, 0] = ref.encode(sign * np.minimum(448, j * 0.6))
        c["cache"].send()
        c["q"][..., 0] = 5.0
        check(c, what=f"climbing {sign}")


def test_nan_where_it_is_seen():
    """A token whose key was not finite makes its requests' rows NaN, and no other's."""
    announce("softmax q8 NaN")
    c = make(2, 2, 4, 2, 64, 32, 32, [50, 50], BF, 22, ALL, 0)
    codes, _ = c["cache"].host["k"]
    codes[c["host"][0, 1], 3, 1, 5] = 127
    c["cache"].send()
    out = run(c, None, out_f32=True)
    assert bool(out[0, :, 2:].isnan().all())
    assert_within(out[0, :, :2], expect(c, 0, 2)[0][:, :2], expect(c, 0, 2)[1][:, :2], FL, "other heads")
    assert_within(out[1], *expect(c, 1, 2), FL, "the other request")


def test_same_bits_and_captured():
    """Twice the same bits; a captured call takes the lengths of each replay."""
    announce("softmax q8 captured")
    c = make(3, 4, 8, 2, 128, 64, 64, [3000, 500, 0], BF, 23, ALL, 0)
    lens, out = i32(c["lens"]), torch.zeros_like(c["q"])
    args = (c["q"], c["k"], c["v"], *c["cache"].args, c["table"], lens, ALL)
    need = hb.workspace_bytes(hb.make_dims(3, 8, 2, 128, 4, 64, hb.HYB_BF16, 1), hb.OP_WINDOW_STEP_Q8,
                              c["table"].shape[1] * 64)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hb.softmax_window_step_paged_q8(*args, out=out, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hb.softmax_window_step_paged_q8(*args, out=out, ws=ws)
    for now in ([3000, 500, 0], [100, 499, 0], [2999, 1, 0], [3000, 500, 0]):
        lens.copy_(i32(now))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        eager = hb.softmax_window_step_paged_q8(*args)
        assert torch.equal(out, eager)
        c["lens"] = now
        for b in range(3):
            assert_within(out[b], *expect(c, b, 4), BF, f"replay {now} {b}")
