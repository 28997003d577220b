"""softmax_window_step_paged_q8 over caches of about one range of keys at most (49152) and more: the arrays
that a range's workgroup keeps of its tiles and pages filled up, requests that must be cut, and blocks of 128
columns, with and without halves, that leave partial rows."""
import pytest
import torch

from _helpers import announce
from _window_ref import assert_within
from test_softmax_q8_gpu import expect, make, run

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32
ALL = 2 ** 31 - 1


def long_among_short(B, L, Hq, Hkv, d, n, dtype):
    """One request of n tokens in pages of 32, the others of none to 99."""
    return make(B, L, Hq, Hkv, d, 32, 32, [n] + [(i * 37) % 100 for i in range(B - 1)], dtype, 50, ALL, 0)


# B, L, Hq, Hkv, d, tokens, dtype.  (A page more than the tokens need belongs to every table.)  49056:
# with that page and the rest of a tile, what one range takes at most.
CASES = [
    (256, 1, 2, 1, 64, 49056, BF), (256, 1, 2, 1, 128, 49000, BF), (256, 2, 2, 1, 64, 49056, FL), (256, 1, 1, 1, 128, 49025, FL),
    (256, 32, 4, 1, 64, 49025, BF), (256, 16, 8, 1, 128, 49025, BF),  # blocks in two halves
    (512, 32, 4, 1, 64, 49025, BF), (512, 32, 4, 1, 128, 49025, BF),  # and without
    (256, 1, 2, 1, 64, 49153, BF), (256, 1, 2, 1, 64, 98305, BF), (256, 1, 1, 1, 128, 60001, FL), (256, 32, 4, 1, 64, 49153, BF),
    (256, 32, 4, 1, 64, 98305, BF), (512, 32, 4, 1, 64, 60001, BF), (512, 32, 4, 1, 128, 50000, BF), (1, 1, 4, 1, 64, 98305, BF),
    (1, 32, 4, 1, 64, 98305, BF)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_long_among_short(case):
    announce(f"softmax q8 ranges {case}")
    B, L, Hq, Hkv, d, n, dtype = case
    c = long_among_short(*case)
    out = torch.full_like(c["q"], 9.0, dtype=FL)
    run(c, None, out=out)
    torch.cuda.synchronize()
    for b in (0, 1, B // 2, B - 1) if B > 1 else (0,):
        assert_within(out[b], *expect(c, b, L), FL, f"{n} tokens, b={b}")
    assert bool(out.isfinite().all())


@pytest.mark.parametrize("B,L,Hq,Hkv,d,dtype", [(256, 1, 2, 1, 64, BF), (256, 1, 2, 1, 64, FL), (256, 32, 4, 1, 64, BF),
                                                (512, 32, 4, 1, 64, BF)])
def test_all_long(B, L, Hq, Hkv, d, dtype):
    """Every request of 98144 tokens, of the same pages, in ranges as long as there are: the first
    against 64 bits, the others, whose queries are the same, equal to it."""
    announce(f"softmax q8 ranges, all long {B} {L} {Hq} {Hkv} {d} {dtype}")
    n = 98144  # with a page more 98176: 6136 of 6144 tiles of two ranges
    c = make(1, L, Hq, Hkv, d, 32, 32, [n], dtype, 51, ALL, 0)
    want = expect(c, 0, L)
    for x in "qkv":
        c[x] = c[x].expand(B, -1, -1, -1).contiguous()
    c["table"] = c["table"].expand(B, -1).contiguous()
    c["lens"] = [n] * B
    out = run(c, None, out_f32=True)
    assert_within(out[0], *want, FL, "all long")
    # (their ranges are cut alike, and so are their sums)
    assert torch.equal(out, out[:1].expand_as(out))
