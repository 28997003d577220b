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
    own = [-(-m // page) for m in lens]
    n = sum(own) + 2
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    table, free = np.zeros((B, per), int), r.permutation(n)
    for b, m in enumerate(own):
        table[b, :m], free = free[:m], free[m:]
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
    if m == 0:
        return None
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
    want = [expect(c, b, L if block is None else min(max(block[b], 0), L)) for b in range(B)]
    for f32 in ([False, True] if dtype == BF else [False]):
        out = torch.full_like(c["q"], 9.0, dtype=FL if f32 else dtype)
        run(c, block, out=out)
        torch.cuda.synchronize()
        for b in range(B):
            m = L if block is None else min(max(block[b], 0), L)
            assert bool((out[b, m:] == 9.0).all()), f"{what}: rows past the block were written"
            if m:
                assert_within(out[b, :m], *want[b], out.dtype, f"{what} b={b}")


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


# Blocks of more workgroups of 32 columns than the chip has CUs, or long caches of several
# requests: most take the kernel of 128 columns.
BLOCKS = [
    (6, 32, 64, 16, 128, 64, 64, [1000, 33, 640, 2048, 0, 31], 96, 32, BF),
    (6, 32, 64, 16, 128, 64, 32, [1000, 33, 640, 2048, 0, 31], 0, 0, BF),
    (6, 32, 64, 16, 64, 32, 32, [1000, 33, 640, 2048, 0, 31], 0, 5, BF),
    (6, 32, 64, 16, 64, 64, 32, [1000, 33, 640, 2048, 1, 32], ALL, 0, BF),
    (8, 29, 36, 12, 128, 32, 32, [95, 64, 0, 1, 32, 33, 300, 128], ALL, 0, BF),  # 3 tiles of columns
    (5, 32, 72, 12, 64, 32, 32, [0, 70, 650, 31, 96], 200, 3, BF),               # 6
    (9, 16, 64, 16, 128, 64, 64, [0, 70, 650, 31, 96, 5, 64, 63, 200], 100, 0, BF),  # 2
    (5, 32, 64, 4, 128, 64, 64, [500, 0, 33, 64, 1], 300, 40, BF),               # 16
    (16, 32, 16, 4, 128, 64, 64, [4000] + [(i * 97) % 300 for i in range(15)], ALL, 0, BF),  # several ranges
    (4, 32, 16, 4, 128, 64, 32, [12000, 1, 5000, 0], ALL, 0, BF),
    (4, 32, 16, 4, 64, 32, 32, [16000, 31, 3000, 64], ALL, 0, BF),
    (16, 32, 16, 4, 64, 64, 64, [16000] + [(i * 71) % 260 for i in range(15)], ALL, 0, BF),
    (9, 32, 128, 32, 128, 64, 32, [0, 1, 31, 32, 33, 200, 65, 129, 400], ALL, 0, BF),  # more workgroups than CUs
    (20, 31, 34, 17, 64, 32, 32, [(i * 29) % 180 for i in range(20)], 70, 9, BF),
    (8, 32, 16, 4, 128, 128, 64, [9000] + [(i * 53) % 200 for i in range(7)], 8500, 70, BF)]
CASES += BLOCKS


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:7]) + f"-{c[7][0]}-{c[8]}-{c[9]}-{str(c[10])[6:]}")
def test_step(case):
    announce(f"softmax q8 {case}")
    B, L, Hq, Hkv, d, page, sb, lens, window, sinks, dtype = case
    c = make(B, L, Hq, Hkv, d, page, sb, lens, dtype, L + d + len(lens), window, sinks)
    check(c, what="whole blocks")
    if L > 1:
        check(c, [[1, L, 0, L - 1, 2][b % 5] for b in range(B)], "active rows")


@pytest.mark.parametrize("d,lens", [(128, [700, 5000, 0, 64]), (64, [3001, 31, 32, 1])])
def test_wide_tables(d, lens):
    """Room for caches of 262144 tokens, of which few are used (the loads past the caches, and many
    ranges that hold nothing)."""
    announce(f"softmax q8 wide tables {d}")
    c = make(4, 1, 16, 4, d, 64, 32, lens, BF, 31, ALL, 0)
    more = torch.full((4, 4096 - c["table"].shape[1]), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    c["table"] = torch.cat([c["table"], more], 1)
    check(c, what="wide tables")


def test_no_cache_at_all():
    """max_pages = 0: the block alone."""
    announce("softmax q8 without pages")
    c = make(2, 8, 4, 2, 64, 32, 32, [0, 0], BF, 3, ALL, 0)
    c["table"] = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    check(c, what="no pages")


@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 1), (32, 32), (33, 31), (64, 33), (100, 64), (5, 200), (0, 64),
                                          (0, 31), (127, 0)])
@pytest.mark.parametrize("L,Hq,Hkv", [(1, 4, 2), (32, 4, 2), (32, 20, 10)])
def test_edges_of_the_window(window, sinks, L, Hq, Hkv):
    announce(f"softmax q8 window {window} {sinks} {L} {Hq}")
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 160, 257]
    check(make(len(lens), L, Hq, Hkv, 64, 32, 32, lens, BF, window + sinks, window, sinks), what=f"{window} {sinks}")


@pytest.mark.parametrize("L,Hq,Hkv", [(4, 4, 1), (32, 258, 129)])
def test_scores_that_climb_and_fall(L, Hq, Hkv):
    """Keys whose scores rise or fall along the prefix by hundreds: the reference moves
    every tile, or never."""
    announce("softmax q8 climbing")
    for sign in (1.0, -1.0):
        c = make(1, L, Hq, Hkv, 64, 32, 32, [700], BF, 21, ALL, 0)
        codes, scales = c["cache"].host["k"]
        scales[:] = 127
        codes[:] = 0
        j = np.arange(700)
        codes[c["host"][0, j // 32], j % 32, :, 0] = ref.encode(sign * np.minimum(448, j * 0.6))[:, None]
        c["cache"].send()
        c["q"][..., 0] = 5.0
        check(c, what=f"climbing {sign}")


@pytest.mark.parametrize("L,G,Hkv", [(2, 2, 2), (32, 2, 65)])
def test_nan_where_it_is_seen(L, G, Hkv):
    """A token whose key was not finite makes its requests' rows NaN, and no other's."""
    announce(f"softmax q8 NaN {L} {Hkv}")
    c = make(2, L, G * Hkv, Hkv, 64, 32, 32, [50, 50], BF, 22, ALL, 0)
    codes, _ = c["cache"].host["k"]
    codes[c["host"][0, 1], 3, 1, 5] = 127
    c["cache"].send()
    out = run(c, None, out_f32=True)
    assert bool(out[0, :, 2:4].isnan().all())
    (o, e), keep = expect(c, 0, L), [h for h in range(G * Hkv) if h // G != 1]
    assert_within(out[0][:, keep], o[:, keep], e[:, keep], FL, "other heads")
    assert_within(out[1], *expect(c, 1, L), FL, "the other request")


@pytest.mark.parametrize("B,L,Hq,Hkv", [(3, 4, 8, 2), (20, 32, 16, 4)])
def test_same_bits_and_captured(B, L, Hq, Hkv):
    """Twice the same bits; a captured call takes the lengths of each replay."""
    announce(f"softmax q8 captured {B} {L}")
    more = [0] * (B - 3)
    c = make(B, L, Hq, Hkv, 128, 64, 64, [3000, 500, 0] + more, BF, 23, ALL, 0)
    lens, out = i32(c["lens"]), torch.zeros_like(c["q"])
    args = (c["q"], c["k"], c["v"], *c["cache"].args, c["table"], lens, ALL)
    need = hb.workspace_bytes(hb.make_dims(B, Hq, Hkv, 128, L, 64, hb.HYB_BF16, 1), hb.OP_WINDOW_STEP_Q8,
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
        now = now + more
        lens.copy_(i32(now))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        eager = hb.softmax_window_step_paged_q8(*args)
        assert torch.equal(out, eager)
        c["lens"] = now
        for b in range(3):
            assert_within(out[b], *expect(c, b, L), BF, f"replay {now} {b}")
