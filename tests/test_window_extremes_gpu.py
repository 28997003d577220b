"""The windowed softmax where its running references move, where a window or a
number of sinks passes 32 bits, and where it is the whole prefix, against 64
bits as in test_window_gpu.py and test_window_step_gpu.py."""
import numpy as np
import pytest
import torch

import test_window_gpu as W
import test_window_step_gpu as S
from paper_2608_06628_amd import binding as hb

from _window_ref import assert_within, attend, rows64

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


def climb(shape, n):
    """Score added to key j of n: in steps that pass what a reference of the
    weights puts up with (2^8, a score of 5.55), early or late in the sequence,
    down again, and by single keys that leave the others their share."""
    j, top = np.arange(n), (n - 1) // 32
    return {"grow": 6.5 * np.minimum(j // 32, 8), "fall": 6.5 * np.maximum(8 - j // 32, 0),
            "late": 6.5 * np.maximum(j // 32 - (top - 8), 0),
            "spike": np.where(j % 97 == 45, 5.8, 0.0) + np.where(j == n * 3 // 4, 11.0, 0.0)}[shape]


def add_scores(q, k, extra):
    """q [.., d] and k [n, .., d] such that key j's scaled scores rise by extra[j]."""
    d = q.shape[-1]
    up = torch.full((d,), d ** -0.25, dtype=torch.float64)
    up[::3] *= -1.0
    extra = torch.from_numpy(np.asarray(extra, dtype=np.float64)).view(-1, *[1] * (k.dim() - 1))
    return ((q.double().cpu() + up).to(q.dtype).to(q.device),
            (k.double().cpu() + extra * up).to(k.dtype).to(k.device))


@pytest.mark.parametrize("window,sinks", [(1 << 32, 0), ((1 << 40) + 5, 1 << 32), (0, 1 << 31), (16, (1 << 32) + 3)])
def test_sequences_past_32_bits(window, sinks):
    """A window or a number of sinks past 2^31 - 1 sees all there is."""
    W.test_prefill(1, 130, 4, 2, 64, 16, window, sinks, BF, [120])
    W.test_backward(1, 130, 4, 2, 64, 16, window, sinks, BF, [120])


@pytest.mark.parametrize("shape", ["grow", "fall", "late", "spike"])
@pytest.mark.parametrize("B,T,Hq,Hkv,d,L,window,sinks,dtype,lens", [
    (2, 420, 8, 2, 64, 7, 150, 33, BF, [420, 391]), (1, 500, 4, 2, 128, 32, 500, 0, BF, None),
    (1, 700, 2, 2, 64, 16, 64, 300, BF, None), (1, 1100, 4, 1, 128, 32, 1100, 0, BF, None),
    (1, 1057, 2, 1, 64, 1, 1040, 3, BF, None), (1, 1100, 2, 1, 64, 1, 1100, 0, FL, None), (2, 400, 4, 2, 128, 9, 90, 40, FL, None)])
def test_references_over_sequences(monkeypatch, shape, B, T, Hq, Hkv, d, L, window, sinks, dtype, lens):
    """Scores that climb or fall along the keys by far more than the slack of a row's
    reference: sums of keys already seen are scaled down in the middle of a list,
    and the halves of a list end on different references."""
    plain = W.make

    def climbing(*args):
        c = plain(*args)
        for b in range(B):
            c["q"][b], c["k"][b] = add_scores(c["q"][b], c["k"][b], climb(shape, T))
        return c

    monkeypatch.setattr(W, "make", climbing)
    W.test_prefill(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens)
    W.test_backward(B, T, Hq, Hkv, d, L, window, sinks, dtype, lens)


@pytest.mark.parametrize("window,sinks", [(1 << 32, 0), ((1 << 40) + 5, 1 << 32), (3, (1 << 32) + 1)])
def test_steps_past_32_bits(window, sinks):
    """A window or a number of sinks past 2^31 - 1 sees all there is."""
    c = S.make(2, 5, 8, 2, 64, 32, [200, 33], BF, 8)
    S.hide(c, window, sinks)
    S.check(c, window, sinks, what="past 32 bits")


@pytest.mark.parametrize("shape", ["grow", "fall", "late", "spike"])
@pytest.mark.parametrize("B,L,Hq,Hkv,d,page,lens,window,sinks,dtype", [
    (3, 1, 16, 4, 128, 64, [1500, 700, 90], 1200, 40, BF),   # one token: four waves take the tiles in turn
    (2, 5, 8, 8, 64, 32, [900, 390], 800, 0, BF),            # a head per KV head
    (1, 1, 16, 4, 128, 64, [9000], 8000, 70, BF),            # ranges that are merged
    (70, 32, 8, 2, 64, 32, [i * 17 % 900 for i in range(70)], 700, 33, BF),  # blocks, in two halves
    (70, 32, 4, 2, 128, 32, [i * 17 % 900 for i in range(70)], 700, 33, BF),
    (40, 32, 32, 4, 128, 64, [i * 31 % 900 for i in range(40)], 700, 33, BF),  # eight heads: the copy ring
    (60, 32, 24, 8, 64, 32, [i * 31 % 700 for i in range(60)], 500, 40, BF),   # three: staged in registers
    (3, 21, 8, 4, 64, 32, [700, 390, 64], 600, 5, FL),
    (2, 1, 4, 1, 128, 64, [5000, 900], 4500, 64, FL)])
def test_references_over_a_cache(shape, B, L, Hq, Hkv, d, page, lens, window, sinks, dtype):
    """Scores that climb or fall along the cache by far more than the slack of a
    query's reference: waves, halves and ranges end on different ones."""
    c = S.make(B, L, Hq, Hkv, d, page, lens, dtype, B + L)
    for b, n in enumerate(lens):
        j = np.arange(n)
        at = c["table"][b].cpu().numpy()[j // page].astype(np.int64) * page + j % page
        rows = torch.from_numpy(at).cuda()
        pool = c["kp"].view(-1, Hkv, d)
        keys = torch.cat([pool[rows], c["k"][b]])
        c["q"][b], keys = add_scores(c["q"][b], keys, climb(shape, n + L))
        pool[rows], c["k"][b] = keys[:n], keys[n:]
    S.hide(c, window, sinks)
    S.check(c, window, sinks, what=shape)


@pytest.mark.parametrize("B,L,Hq,Hkv,d,lens", [
    (3, 32, 16, 4, 128, [700, 64, 2000]), (40, 32, 16, 4, 64, [i * 53 % 2000 for i in range(40)]),
    (2, 1, 8, 2, 128, [1990, 333]), (24, 32, 16, 2, 128, [i * 83 % 2000 for i in range(24)])])
def test_all_of_the_cache_by_row(B, L, Hq, Hkv, d, lens):
    """A window of the whole prefix and softmax_prefix_step_paged, both within what
    the weights' roundings allow of each row."""
    c = S.make(B, L, Hq, Hkv, d, 64, lens, BF, 5)
    S.check(c, 2048, 0, what="window")
    out = hb.softmax_prefix_step_paged(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], out_f32=True)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        row = c["table"][b].cpu().numpy()[np.arange(n) // 64].astype(np.int64) * 64 + np.arange(n) % 64
        kc, vc = (rows64(p.view(-1, Hkv, d)[torch.from_numpy(row).cuda()]) for p in (c["kp"], c["vp"]))
        kb, vb = np.concatenate([kc, rows64(c["k"][b])]), np.concatenate([vc, rows64(c["v"][b])])
        for h in range(0, Hq, 3):
            g = h * Hkv // Hq
            o, _, err, _ = attend(rows64(c["q"][b, :, h]), kb[:, g], vb[:, g], np.ones((L, len(kb)), bool), True)
            assert_within(out[b, :, h], o, err * 1.001 + 2.0 ** -8 * 1.01 * np.abs(o), FL, f"prefix b={b} h={h}")
