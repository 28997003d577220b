"""The 8-bit cache with scales that its own write does not leave: zeroed pools, whose scales are
2^-127, and bytes below 10, as another writer of the format may leave them."""
import numpy as np
import pytest
import torch

from paper_2608_06628_amd import binding as hb

import _cache_ref as ref
from _helpers import announce
from test_kv_q8_gpu import same
from test_softmax_q8_gpu import check, make, run

pytestmark = pytest.mark.gpu
BF, FL = torch.bfloat16, torch.float32
ALL = 2 ** 31 - 1

LENS = [1, 33, 70, 0, 200, 31]
SHAPES = [  # B, L, Hq, Hkv, d, dtype: tokens, blocks by 32 columns, by 128, by 128 without halves
    (3, 1, 4, 2, 64, BF), (3, 1, 8, 2, 128, BF), (3, 1, 4, 2, 64, FL), (2, 5, 4, 1, 128, FL), (3, 32, 4, 2, 64, BF),
    (6, 32, 64, 16, 64, BF), (6, 32, 64, 16, 128, BF), (6, 32, 160, 80, 64, BF), (6, 32, 160, 80, 128, BF)]


def cached(shape, window, sinks, byte, what="kv"):
    """A case whose seen scales are all of one byte, in K or V or both."""
    B, L, Hq, Hkv, d, dtype = shape
    c = make(B, L, Hq, Hkv, d, 64, 32, LENS[:B], dtype, 40 + byte, window, sinks)
    for x in what:
        scales = c["cache"].host[x][1]
        scales[scales != 255] = byte
    c["cache"].send()
    return c


@pytest.mark.parametrize("byte,what", [(0, "k"), (0, "v"), (0, "kv"), (1, "kv"), (9, "k")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step(shape, byte, what):
    """Tiles that the lengths and the window cut, under the least scales there are."""
    announce(f"softmax q8 scale byte {byte} of {what}: {shape}")
    check(cached(shape, ALL, 0, byte, what), what=f"byte {byte} of {what}")
    check(cached(shape, 40, 3, byte, what), what=f"byte {byte} of {what}, a window")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step_over_zeroed_pools(shape):
    """A pool as torch.zeros leaves it: every cached key and value is zero."""
    announce(f"softmax q8 zeroed pools: {shape}")
    for window, sinks in ((ALL, 0), (40, 3)):
        c = cached(shape, window, sinks, 0)
        for x in "kv":
            for t in c["cache"].host[x]:
                t[:] = 0
        c["cache"].send()
        check(c, what="zeroed pools")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_values_of_the_least_scale(shape):
    """Even weights (q is zero) over 64 tokens of which one is the block's, zero: the mean of codes times
    2^-127, exact up to the order of a sum of numbers of 16 bits and a reciprocal (2 steps of fp32)."""
    B, _, Hq, Hkv, d, dtype = shape
    L = shape[1]
    n = 64 - L
    c = make(B, L, Hq, Hkv, d, 64, 32, [n] * B, dtype, 7, ALL, 0)
    announce(f"softmax q8 values of the least scale: {shape}")
    codes, scales = c["cache"].host["v"]
    codes[:] = np.random.RandomState(8).randint(0x40, 0x7f, codes.shape)  # 2 .. 448, so that 2^-127 of it is normal
    scales[:] = 0
    c["cache"].send()
    c["q"].zero_(), c["v"].zero_()
    out = run(c, None, out_f32=True).double().cpu().numpy()
    values = ref.values(*c["cache"].host["v"])
    for b in range(B):
        j = np.arange(n)
        want = values[c["host"][b, j // 64], j % 64].sum(0) / 64
        want = want.repeat(Hq // Hkv, 0)[None]
        assert np.abs(out[b] - want).max() <= 2.0 ** -22 * np.abs(want).max()


def every_byte():
    """A pool of 256 pages of 32 rows with every code, page n under the scale byte n, and its values."""
    codes = np.arange(2048).astype(np.uint8).reshape(1, 32, 1, 64).repeat(256, 0)
    scales = np.arange(256).astype(np.uint8).reshape(256, 1, 1)
    return codes, scales, torch.from_numpy(ref.values(codes, scales)).flatten(0, 1)


@pytest.mark.parametrize("dtype", [BF, FL], ids=str)
def test_read(dtype):
    """Every code under every scale but 255: the value, rounded to nearest even where bf16 has fewer bits
    (subnormal numbers), an infinity where the type ends."""
    announce(f"read every scale byte {dtype}")
    codes, scales, values = every_byte()
    pool = torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn)
    bytes_ = torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    k, v = hb.kv_pages_q8_read(pool, pool, bytes_, bytes_, i32([list(range(255))]), i32([0]), i32([0, 255 * 32]),
                               tokens=255 * 32, dtype=dtype)
    want = values[:255 * 32].float().to(dtype)
    for t in (k, v):
        assert torch.equal(t.isnan().cpu(), want.isnan())
        assert torch.equal(torch.nan_to_num(t.cpu(), 3.0, 5.0, -5.0), torch.nan_to_num(want, 3.0, 5.0, -5.0))


@pytest.mark.parametrize("old", [0, 1, 9, 10, 253, 254])
@pytest.mark.parametrize("dtype,H,d,page,sb", [(BF, 2, 128, 64, 32), (FL, 3, 64, 64, 64), (BF, 1, 64, 256, 256),
                                               (FL, 2, 128, 1024, 512)])
def test_write_goes_on(dtype, H, d, page, sb, old):
    """Blocks that hold rows under any scale and go on: those rows are rounded again to the new scale
    wherever that is larger, whatever the old one was."""
    announce(f"write goes on from scale byte {old}: {dtype} {H} {d} {page} {sb}")
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    held, new = [1, sb - 1, 5, sb // 2, 0, 17], [1, 1, sb, 3, 2, 0]
    B = len(held)
    table = np.random.RandomState(9).permutation(2 * B).reshape(B, 2).astype(np.int32)
    start = np.concatenate([[0], np.cumsum(new)])
    g = torch.Generator().manual_seed(old)
    for size in (0.0, 1e-36, 1.0, 1e30):
        cache = ref.Cache(2 * B, page, sb, H, d, 10)
        for x in "kv":
            cache.host[x][1][:] = old
        cache.send()
        k, v = ((torch.randn(int(start[-1]), H, d, generator=g) * size).to(dtype).cuda() for _ in "kv")
        hb.kv_pages_q8_write(k, v, *cache.args, i32(table), i32(held), i32(start))
        torch.cuda.synchronize()
        for x, t in (("k", k), ("v", v)):
            ref.write(*cache.host[x], t.double().cpu().numpy(), table, held, start.copy())
            same(cache.codes(x), cache.host[x], f"{x}, new rows of {size}")


@pytest.mark.parametrize("dtype", [BF, FL], ids=str)
def test_read_not_a_number(dtype):
    """Byte 255 is the format's NaN: so is every value under it."""
    announce(f"read scale byte 255 {dtype}")
    codes, scales, _ = every_byte()
    pool = torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn)
    bytes_ = torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    k, v = hb.kv_pages_q8_read(pool, pool, bytes_, bytes_, i32([[255]]), i32([0]), i32([0, 32]), tokens=32, dtype=dtype)
    assert bool(k.isnan().all()) and bool(v.isnan().all())


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step_not_a_number(shape, what):
    """A seen block of scale byte 255 makes its request's rows NaN at the query heads of its KV head,
    whatever its codes and the queries are, and no others."""
    B, L, Hq, Hkv, d, dtype = shape
    announce(f"softmax q8 scale byte 255 of {what}: {shape}")
    c = cached(shape, ALL, 0, 127)
    codes, scales = c["cache"].host[what]
    g, page = min(1, Hkv - 1), c["host"][1, 0]  # request 1 has 33 tokens: two blocks, the second cut
    scales[page, 1, g] = 255
    codes[page, 32, g] = np.where(np.arange(d) % 2, 0, 0x38 + 128 * (np.arange(d) // 2 % 2))
    c["cache"].send()
    out = run(c, None, out_f32=True)
    heads = torch.arange(Hq) // (Hq // Hkv) == g
    assert bool(out[1][:, heads].isnan().all())
    assert not bool(out[1][:, ~heads].isnan().any())
    assert not bool(out[[b for b in range(B) if b != 1]].isnan().any())


def test_write_goes_on_from_not_a_number():
    """A block that holds rows under scale byte 255, which are NaN, and goes on keeps it: no NaN becomes a
    number."""
    announce("write goes on from scale byte 255")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    for dtype, sb in ((BF, 32), (FL, 64), (BF, 256)):
        cache = ref.Cache(2, sb, sb, 2, 64, 11)
        for x in "kv":
            cache.host[x][1][:] = 255
        cache.send()
        k = torch.ones(sb, 2, 64, dtype=dtype, device="cuda")
        hb.kv_pages_q8_write(k, k, *cache.args, i32([[0, 1]]), i32([5]), i32([0, sb]))
        k2, v2 = hb.kv_pages_q8_read(*cache.args, i32([[0, 1]]), i32([0]), i32([0, sb + 5]), tokens=sb + 5, dtype=FL)
        for t in (k2, v2):
            assert bool(t[:sb].isnan().all()) and bool((t[sb:] == 1.0).all())  # (the second block starts over)
