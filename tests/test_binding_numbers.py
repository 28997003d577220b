"""Numbers past 32 bits in the binding's calls: those that mean "all of it" are
taken as that, the others are refused; none arrives with its high bits lost.
The library is a recorder here, and the tensors are the host's."""
import ctypes

import pytest
import torch

from paper_2608_06628_amd import binding as hb

MOST = 2 ** 31 - 1


class Recorder:
    """A library whose functions note their numbers as a C int32 would hold them."""

    def __init__(self):
        self.calls = {}

    def __getattr__(self, name):
        def call(*args):
            self.calls[name] = [ctypes.c_int32(a).value if isinstance(a, int) else a for a in args]
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(hb, "load", lambda: lib)
    monkeypatch.setattr(hb, "_raw_stream", lambda dev: None)
    return lib


def call(f, *args, **kw):
    return f.__wrapped__(-1, *args, **kw)  # (-1: the device of a host tensor)


t = torch.zeros(2, 8, 4, 64)
lens = torch.zeros(2, dtype=torch.int32)
table = torch.zeros(2, 3, dtype=torch.int32)
pool = torch.zeros(5, 32, 4, 64)
CALLS = {  # the place of window and n_sinks in the library's call
    "softmax_window_step_paged": (11, lambda w, s, **kw: call(hb.softmax_window_step_paged, t, t, t, pool, pool, table, lens,
                                                              w, s, **kw)),
    "softmax_window_prefill": (2, lambda w, s, b=4: call(hb.softmax_window_prefill, t, t, t, b, w, s)),
    "softmax_window_backward": (2, lambda w, s, b=4: call(hb.softmax_window_backward, t, t, t, t, torch.zeros(2, 4, 8), t, b,
                                                          w, s)),
}


@pytest.mark.parametrize("name", CALLS)
def test_windows(lib, name):
    at, f = CALLS[name]
    for given, taken in ((0, 0), (5, 5), (MOST, MOST), (MOST + 1, MOST), (1 << 32, MOST), ((1 << 40) + 5, MOST),
                         (10 ** 30, MOST), (-1, -1), (-(1 << 32), -1), (-(1 << 32) + 5, -1)):
        f(given, 3)
        assert lib.calls[name][at:at + 2] == [taken, 3], given
        f(3, given)
        assert lib.calls[name][at:at + 2] == [3, taken], given
        if "hybrid_workspace_bytes" in lib.calls and given >= 0:
            assert 0 <= lib.calls["hybrid_workspace_bytes"][2] <= 96  # (the table's tokens at most)
    with pytest.raises(TypeError):
        f(4.0, 0)


@pytest.mark.parametrize("block", [(1 << 32) + 4, 1 << 31, -(1 << 32) + 4])
def test_blocks(lib, block):
    for name in ("softmax_window_prefill", "softmax_window_backward"):
        with pytest.raises(ValueError):
            CALLS[name][1](3, 3, block)
    with pytest.raises(ValueError):
        hb.make_dims(1, 4, 4, 64, block, 64, hb.HYB_F32, 1)


def test_plan(lib):
    plan = lambda page, most, free=lens: call(hb.kv_pages_plan, lens, lens, table, free, page, most)
    plan(32, 7)
    assert lib.calls["kv_pages_plan"][:5] == [2, 3, 32, 2, 7]
    for page, most in ((32, 1 << 32), (32, (1 << 32) + 7), (32, MOST + 1), (32, -1), ((1 << 32) + 32, 7), (-(1 << 32) + 32, 7)):
        with pytest.raises(ValueError):
            plan(page, most)
    plan(32, 7, lens[:1].expand(1 << 33)[:0])
    assert lib.calls["kv_pages_plan"][3] == 0


def test_long_tables(lib):
    """A table of more than 2^31 entries per request (its memory is not there)."""
    wide = torch.zeros(2, 1, dtype=torch.int32).expand(2, (1 << 32) + 3)
    with pytest.raises(ValueError):
        call(hb.kv_pages_plan, lens, lens, wide, lens, 32, 7)
