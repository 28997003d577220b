"""softmax_window_step_paged against 64 bits: what of the cache is seen, and
that nothing else plays a part."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import assert_within, attend, rows64

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def make(B, L, Hq, Hkv, d, page, lens, dtype, seed, spare=3):
    g = torch.Generator().manual_seed(seed)
    per = -(-max(list(lens) + [1]) // page) + 1
    n = B * per + spare
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    table = torch.randperm(n, generator=g)[:B * per].to(torch.int32).view(B, per).cuda()
    return dict(q=rnd(B, L, Hq, d), k=rnd(B, L, Hkv, d), v=rnd(B, L, Hkv, d), kp=rnd(n, page, Hkv, d),
                vp=rnd(n, page, Hkv, d), table=table, lens=torch.tensor(list(lens), dtype=torch.int32).cuda(), page=page)


def seen(n, window, sinks):
    j = np.arange(n)
    return j[(j >= n - window) | (j < sinks)]


def hide(c, window, sinks):
    """NaN in every cached row that is not seen; entries of the table that are
    not read name pages far outside the pool."""
    for pool in (c["kp"], c["vp"]):
        keep = torch.zeros(pool.shape[:2], dtype=torch.bool)
        for b, n in enumerate(c["lens"].tolist()):
            j = seen(n, window, sinks)
            keep[c["table"][b].cpu()[j // c["page"]].long(), j % c["page"]] = True
        pool[~keep.cuda()] = float("nan")
    for b, n in enumerate(c["lens"].tolist()):
        w0 = max(0, n - window)
        e = np.arange(c["table"].shape[1])
        read = (e < -(-min(sinks, n) // c["page"])) | ((e >= w0 // c["page"]) & (e < -(-n // c["page"])))
        c["table"][b, torch.from_numpy(~read).cuda()] = 2 ** 31 - 1


def check(c, window, sinks, block=None, what=""):
    B, L, Hq, d = c["q"].shape
    Hkv, page = c["k"].shape[2], c["page"]
    dtype = c["q"].dtype
    bl = None if block is None else torch.tensor(block, dtype=torch.int32).cuda()
    for f32 in ([False, True] if dtype == BF else [False]):
        out = torch.full_like(c["q"], 9.0, dtype=FL if f32 else dtype)
        hb.softmax_window_step_paged(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], window, sinks,
                                     block_len=bl, out=out)
        torch.cuda.synchronize()
        for b, n in enumerate(c["lens"].tolist()):
            m = L if block is None else min(max(block[b], 0), L)
            assert bool((out[b, m:] == 9.0).all()), f"{what}: rows past the block were written"
            if m == 0:
                continue
            j = seen(n, window, sinks)
            row = c["table"][b].cpu().numpy()[j // page].astype(np.int64) * page + j % page
            kc, vc = (rows64(p.view(-1, Hkv, d)[torch.from_numpy(row).cuda()]) for p in (c["kp"], c["vp"]))
            kb, vb = np.concatenate([kc, rows64(c["k"][b, :m])]), np.concatenate([vc, rows64(c["v"][b, :m])])
            for h in range(Hq):
                g = h * Hkv // Hq
                o, _, err, _ = attend(rows64(c["q"][b, :m, h]), kb[:, g], vb[:, g], np.ones((m, len(kb)), bool),
                                      dtype == BF)
                # the sum of the weights is over the rounded ones too
                assert_within(out[b, :m, h], o, err * 1.001 + (2.0 ** -8 * 1.01 * np.abs(o) if dtype == BF else 0), out.dtype,
                              f"{what} b={b} h={h}")


CASES = [  # B, L, Hq, Hkv, d, page, lens, window, sinks, dtype
    (1, 1, 1, 1, 64, 32, [0], 5, 3, BF),
    (1, 1, 4, 1, 128, 32, [1], 0, 0, BF),
    (5, 1, 16, 4, 128, 64, [4097, 64, 31, 0, 500], 200, 4, BF),
    (4, 32, 16, 4, 128, 64, [1000, 33, 640, 2048], 96, 32, BF),
    (4, 32, 16, 4, 128, 64, [1000, 33, 640, 2048], 0, 0, BF),
    (3, 32, 16, 4, 128, 32, [1000, 999, 640], 0, 33, BF),
    (3, 7, 8, 8, 64, 32, [300, 129, 77], 40, 70, BF),
    (3, 7, 2, 1, 64, 256, [300, 1129, 77], 1, 1, BF),
    (2, 13, 16, 2, 64, 64, [800, 5], 127, 0, BF),
    (2, 13, 16, 2, 128, 64, [800, 290], 33, 65, BF),
    (2, 32, 12, 4, 128, 64, [700, 90], 65, 31, BF),
    (3, 17, 5, 1, 64, 32, [64, 400, 96], 32, 64, BF),
    (2, 21, 8, 4, 64, 32, [350, 97], 50, 5, FL),
    (3, 1, 4, 4, 128, 64, [0, 700, 65], 64, 64, FL),
    (2, 32, 6, 2, 128, 32, [256, 95], 2 ** 31 - 1, 0, FL),
    (2, 32, 16, 4, 128, 32, [256, 95], 2 ** 31 - 1, 2 ** 31 - 1, BF),
    (70, 4, 4, 2, 64, 32, [i * 13 % 400 for i in range(70)], 64, 10, BF),
]


@pytest.mark.parametrize("B,L,Hq,Hkv,d,page,lens,window,sinks,dtype", CASES)
def test_step(B, L, Hq, Hkv, d, page, lens, window, sinks, dtype):
    announce(f"window step {B} {L} {Hq} {Hkv} {d} {page} {lens[:5]} {window} {sinks} {dtype}")
    c = make(B, L, Hq, Hkv, d, page, lens, dtype, B * 100 + L)
    hide(c, window, sinks)
    check(c, window, sinks, what="step")


@pytest.mark.parametrize("B,Hq,Hkv,d,dtype,window,sinks", [
    (6, 16, 4, 128, BF, 100, 4), (6, 3, 3, 64, FL, 33, 40), (6, 8, 1, 64, BF, 0, 0), (6, 10, 2, 128, BF, 700, 1)])
def test_blocks_of_every_length(B, Hq, Hkv, d, dtype, window, sinks):
    announce(f"window step ragged {Hq} {Hkv} {d}")
    c = make(B, 32, Hq, Hkv, d, 32, [900, 64, 0, 31, 512, 200], dtype, 7)
    hide(c, window, sinks)
    block = [5, 0, 1, 32, 40, -3]
    for b, m in enumerate(block):
        for n in ("q", "k", "v"):
            c[n][b, min(max(m, 0), 32):] = float("nan")
    check(c, window, sinks, block, "ragged")


def test_long_cache_in_ranges():
    """A window of many tiles is cut into ranges, with the sinks' tiles and the
    skipped ones inside the first."""
    announce("window step long")
    c = make(2, 4, 8, 2, 128, 64, [9000, 6001], BF, 17)
    hide(c, 5000, 100)
    check(c, 5000, 100, what="long")


def test_every_boundary():
    """Window and sinks ends at every place of a tile and a page."""
    announce("window step boundaries")
    for window in (1, 31, 32, 33, 63, 64, 65):
        for sinks in (0, 1, 32, 63, 65):
            c = make(2, 3, 2, 1, 64, 64, [200 + window, 131], BF, window)
            hide(c, window, sinks)
            check(c, window, sinks, what=f"{window} {sinks}")


def test_all_of_the_cache():
    """A window of the whole prefix is softmax_prefix_step_paged, within the
    roundings of both."""
    c = make(3, 32, 16, 4, 128, 64, [700, 64, 2000], BF, 5)
    a = hb.softmax_window_step_paged(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], 2048, 0, out_f32=True)
    b = hb.softmax_prefix_step_paged(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], out_f32=True)
    torch.cuda.synchronize()
    # each weight is off by 2^-8 at most in either
    assert float((a - b).abs().max()) <= 4 * 2.0 ** -8 * float(c["vp"].abs().max())


def test_no_pages():
    c = make(2, 8, 4, 2, 64, 32, [0, 0], BF, 9)
    out = hb.softmax_window_step_paged(c["q"], c["k"], c["v"], c["kp"][:0], c["vp"][:0], c["table"][:, :0], c["lens"], 10, 2)
    ref = hb.softmax_window_step_paged(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], 10, 2)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_streams_and_replays():
    """A side stream gives the same bits; a captured call sees each replay's
    lengths; two graphs keep workspaces of their own."""
    c = make(4, 2, 16, 4, 128, 64, [3000, 2500, 70, 0], BF, 31)
    args = lambda: (c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], 1500, 4)
    want = hb.softmax_window_step_paged(*args())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hb.softmax_window_step_paged(*args(), stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = hb.softmax_window_step_paged(*args())
        graphs.append((graph, out))
    for lens in ([3000, 2500, 70, 0], [1, 3000, 1600, 33], [64, 64, 64, 64]):
        c["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = hb.softmax_window_step_paged(*args())
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for _, o in graphs), lens


@pytest.mark.parametrize("B,L,Hq,Hkv,d,window,sinks", [
    (70, 32, 16, 4, 128, 90, 4), (70, 20, 8, 4, 64, 300, 33), (40, 32, 32, 8, 128, 64, 0), (33, 32, 16, 8, 128, 500, 1),
    (9, 24, 12, 4, 128, 200, 4), (40, 9, 32, 4, 64, 100, 2), (3, 11, 16, 4, 128, 1500, 7), (130, 3, 10, 2, 128, 40, 5)])
def test_batches(B, L, Hq, Hkv, d, window, sinks):
    """Batches that fill the chip, and few requests whose heads are spread over
    it, with requests of every length and one that is empty."""
    announce(f"window step batch {B} {L} {Hq} {Hkv} {d}")
    lens = [i * 37 % 700 for i in range(B)]
    c = make(B, L, Hq, Hkv, d, 32, lens, BF, B + L)
    hide(c, window, sinks)
    check(c, window, sinks, [(i * 7) % (L + 1) for i in range(B)], what="batch")
