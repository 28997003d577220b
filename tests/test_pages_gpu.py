"""kv_pages_plan against a plain loop over requests and tokens."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

from _helpers import announce

pytestmark = pytest.mark.gpu


def plain(prefix, new, table, free, page, max_tokens):
    """The plan one token at a time."""
    B, max_pages = table.shape
    table = table.copy()
    cap = max_pages * page
    slots, pos = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int64)
    start, taken, t = [0], 0, 0
    for b in range(B):
        p = min(max(int(prefix[b]), 0), cap)
        n = max(int(new[b]), 0)
        for e in range(-(-p // page), -(-min(p + n, cap) // page)):
            table[b, e] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(min(n, max(0, max_tokens - t))):
            pos[t + i] = p + i
            if p + i < cap and table[b, (p + i) // page] >= 0:
                s = int(table[b, (p + i) // page]) * page + (p + i) % page
                slots[t + i] = s if s < 2 ** 31 else -1
        t = min(t + n, 2 ** 31 - 1)
        start.append(t)
    return slots, pos, np.array(start), np.array([min(taken, len(free)), max(taken - len(free), 0)]), table


def check(prefix, new, table, free, page, max_tokens, what):
    announce(f"pages {what}")
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    tab = i32(table)
    got = hb.kv_pages_plan(i32(prefix), i32(new), tab, i32(free), page, max_tokens)
    torch.cuda.synchronize()
    want = plain(prefix, new, np.asarray(table), np.asarray(free), page, max_tokens)
    for g, w, n in zip(got + (tab,), want, ("slots", "positions", "token_start", "counts", "page_table")):
        assert np.array_equal(g.cpu().numpy().astype(np.int64), w), (what, n)


@pytest.mark.parametrize("B,page,most,cached,free,extra", [
    (1, 32, 1, 0, 4, 0), (1, 64, 1, 64, 1, 5), (3, 32, 40, 100, 50, 7), (64, 64, 32, 500, 200, 0),
    (65, 16, 70, 90, 100, 3), (257, 32, 9, 64, 30, 100), (300, 1, 5, 9, 5000, 1), (1000, 256, 33, 3000, 4000, 0),
    (4096, 32, 3, 60, 2000, 11), (5, 32, 3000, 100, 600, 2)])
def test_plan(B, page, most, cached, free, extra):
    rng = np.random.default_rng(B + page)
    prefix, new = rng.integers(0, cached + 1, B), rng.integers(0, most + 1, B)
    max_pages = -(-(cached + most) // page)
    order = rng.permutation(B * max_pages + free)
    table = order[:B * max_pages].reshape(B, max_pages)
    held = -(-prefix // page)
    table = np.where(np.arange(max_pages)[None] < held[:, None], table, -1)
    check(prefix, new, table, order[B * max_pages:], page, int(new.sum()) + extra, (B, page, most))


def test_edges():
    t = np.array([[5, 6, -1, -1], [7, -1, -1, -1], [8, 9, 10, 11]])
    # a full request, nothing new anywhere, lengths below zero and past the table
    check([64, 3, 128], [0, 0, 0], t, [1, 2, 3], 32, 8, "nothing new")
    check([64, -7, 10 ** 9], [-5, 3, 4], t, [1, 2, 3], 32, 8, "clamped lengths")
    check([60, 20, 100], [70, 200, 500], t, [1, 2, 3, 4, 12, 13], 32, 800, "past the table")
    check([60, 20, 100], [70, 200, 500], t, [], 32, 800, "no free page")
    check([60, 20, 100], [70, 200, 500], t, [1], 32, 50, "fewer rows than tokens")
    check([60, 20, 100], [70, 2 ** 31 - 1, 2 ** 31 - 1], t, [1, 2], 32, 100, "sums past 31 bits")
    check([60, 20, 100], [5, 5, 5], t, [1], 32, 0, "no rows")
    # page numbers that name no row: negative and too large
    check([33, 1, 3], [2, 2, 2], [[5, -9], [2 ** 31 - 1, 0], [2 ** 26 - 1, 0]], [3], 32, 6, "bad pages")
    check([0], [3], np.zeros((1, 0)), [1], 32, 4, "no table")


def test_no_requests():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    s, p, start, c = hb.kv_pages_plan(e, e, e.view(0, 4), e, 32, 3)
    assert s.tolist() == [-1] * 3 and p.tolist() == [0] * 3 and start.tolist() == [0] and c.tolist() == [0, 0]


def test_replay_plans_from_new_lengths():
    dev = "cuda"
    prefix = torch.tensor([10, 40, 0], dtype=torch.int32, device=dev)
    new = torch.tensor([4, 30, 2], dtype=torch.int32, device=dev)
    table = torch.full((3, 4), -1, dtype=torch.int32, device=dev)
    free = torch.arange(20, dtype=torch.int32, device=dev)
    held = torch.tensor([[50, -1, -1, -1], [51, 52, -1, -1], [-1, -1, -1, -1]], dtype=torch.int32, device=dev)
    table.copy_(held)
    hb.kv_pages_plan(prefix, new, table, free, 32, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = hb.kv_pages_plan(prefix, new, table, free, 32, 64)
    for i in range(3):
        prefix.copy_(torch.tensor([10 + i, 40 + 11 * i, 0], dtype=torch.int32))
        new.copy_(torch.tensor([30 * i, 1 + i, 40], dtype=torch.int32))
        table.copy_(held)
        graph.replay()
        torch.cuda.synchronize()
        want = plain(prefix.tolist(), new.tolist(), held.cpu().numpy(), free.tolist(), 32, 64)
        for g, w in zip(got + (table,), want):
            assert np.array_equal(g.cpu().numpy().astype(np.int64), w), i
