"""A serving loop (page plan, norm and rotation into the pages, windowed step) on
bf16, held to the softmax's own roundings."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce
from _window_ref import assert_within, attend, rows64

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32


@pytest.mark.parametrize("Hq,Hkv,d,L,window,sinks", [(16, 4, 128, 1, 40, 4), (8, 2, 128, 32, 64, 0), (4, 4, 64, 7, 31, 5)])
def test_serving_of_rounded_rows(Hq, Hkv, d, L, window, sinks):
    """bf16: a serving loop with ragged blocks, against 64 bits on the rounded
    queries and keys themselves (those of the whole sequence, normalised and
    rotated in one call), so that only the softmax's own roundings are allowed
    and one key more or less shows."""
    announce(f"serving of rounded rows {Hq} {Hkv} {d} {L}")
    page, max_pages, B, steps = 32, 8, 3, 4
    g = torch.Generator().manual_seed(L + d)
    held, blocks = [66, 31, 0], [[L, max(L - 2, 0), 1], [L, 0, L], [1, L, L], [L, L, max(L // 2, 1)]]
    n_tok = [h + sum(s[b] for s in blocks) for b, h in enumerate(held)]
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(BF).cuda() for _ in range(2)]
    freq = (1e4 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).cuda()
    raw, whole = [], []  # per request its projections' q, k, v, and what the attention should see
    for n in n_tok:
        q, k, v = (torch.randn(n, h, d, generator=g).mul(1.3).to(BF).cuda() for h in (Hq, Hkv, Hkv))
        pos = torch.arange(n, dtype=torch.int32, device="cuda")
        raw.append((q, k, v))
        whole.append([rows64(t) for t in (*hb.hybrid_qk_norm_rope(q, k, freq, pos, *w), v)])
    kp = torch.full((B * max_pages, page, Hkv, d), float("nan"), dtype=BF, device="cuda")
    vp = kp.clone()
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(B * max_pages, generator=g).to(torch.int32).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()

    def cached(sizes):
        nonlocal free
        lens = i32(held)
        slots, pos, start, counts = hb.kv_pages_plan(lens, i32(sizes), table, free, page, sum(sizes) + 3)
        rows = [torch.cat([t[i][a:a + s] for t, a, s in zip(raw, held, sizes)] + [torch.zeros_like(raw[0][i][:3])])
                for i in range(3)]
        q, k = hb.hybrid_qk_norm_rope_paged(*rows, freq, pos, slots, kp, vp, *w, want_k=True)
        taken, missing = counts.tolist()
        assert missing == 0
        free = free[taken:]
        return (q, k, rows[2]), start.tolist(), lens

    prompt, held = held, [0] * B
    cached(prompt)
    held = prompt
    for sizes in blocks[:steps]:
        rows, start, lens = cached(sizes)
        blk = [torch.full((B, L, t.shape[1], d), float("nan"), dtype=BF, device="cuda") for t in rows]
        for b, m in enumerate(sizes):
            for t, s in zip(blk, rows):
                t[b, :m] = s[start[b]:start[b] + m]
        out = hb.softmax_window_step_paged(*blk, kp, vp, table, lens, window, sinks, block_len=i32(sizes), out_f32=True)
        torch.cuda.synchronize()
        for b, m in enumerate(sizes):
            j = np.arange(held[b] + m)
            j = j[(j < sinks) | (j >= held[b] - window)]
            for h in range(Hq if m else 0):
                k, v = (x[j, h * Hkv // Hq] for x in whole[b][1:])
                o, _, err, _ = attend(whole[b][0][held[b]:held[b] + m, h], k, v, np.ones((m, len(j)), bool), True)
                # (the sum of the weights may be over the rounded ones too)
                assert_within(out[b, :m, h], o, err * 1.001 + 2.0 ** -8 * 1.01 * np.abs(o), FL, f"b={b} h={h}")
        held = [a + m for a, m in zip(held, sizes)]
