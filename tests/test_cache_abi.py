"""Refusals of the 8-bit cache's write, read and attention: every check runs on the host
before anything is enqueued (the pointers are small fake addresses that no kernel may
see)."""
import ctypes

import pytest
import torch

from paper_2608_06628_amd import binding as hb

from test_operators_abi import A, ODD, Call, dims


def q8(**kw):
    base = dict(tokens=40, batch=2, n_kv_heads=4, head_dim=128, dtype=hb.HYB_BF16, max_pages=3, n_pages=9, page_size=64,
                scale_block=32, k_stride=0, v_stride=0)
    base.update(kw)
    return hb.KvQ8Dims(*[base[n] for n, _ in hb.KvQ8Dims._fields_])


def write(d=None):
    # dims k v k_pages v_pages k_scales v_scales page_table first token_start
    return Call("kv_pages_q8_write", [d or q8()] + [A(i) for i in range(9)] + [None], range(1, 10))


def read(d=None):
    # dims k_pages v_pages k_scales v_scales page_table first token_start k v
    return Call("kv_pages_q8_read", [d or q8()] + [A(i) for i in range(9)] + [None], range(1, 10))


def step(d=None, n_pages=9, page=64, sb=32, max_pages=4, window=100, sinks=4):
    # dims q k v k_pages v_pages k_scales v_scales n_pages page sb table max_pages lens window sinks block_len out ws bytes
    return Call("softmax_window_step_paged_q8",
                [d or dims()] + [A(i) for i in range(7)] + [n_pages, page, sb, A(7), max_pages, A(8), window, sinks, A(9),
                                                            A(10), A(11), 1 << 26, None],
                [1, 2, 3, 4, 5, 6, 7, 11, 13, 16, 17, 18], (16,))


@pytest.mark.parametrize("make", [write, read])
@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), 2), (dict(batch=-1), 2), (dict(n_kv_heads=0), 2), (dict(n_kv_heads=1 << 17), 2), (dict(head_dim=96), 5),
    (dict(dtype=2), 4), (dict(max_pages=-1), 2), (dict(n_pages=0), 2), (dict(page_size=48), 5), (dict(page_size=16), 5),
    (dict(page_size=1 << 17), 5), (dict(scale_block=16), 5), (dict(scale_block=48), 5), (dict(scale_block=128), 5),
    (dict(scale_block=0), 5), (dict(max_pages=1 << 26), 2), (dict(k_stride=504), 2), (dict(v_stride=-512), 2),
    (dict(k_stride=516), 3), (dict(v_stride=1 << 40), 2), (dict(tokens=2 ** 31 - 1, n_kv_heads=4096), 2)])
def test_cache_dims(make, kw, code):
    assert make(q8(**kw))() == code and hb.last_error()


@pytest.mark.parametrize("make", [write, read])
def test_cache_pointers(make):
    c = make()
    assert c.fn(None, *c.args[1:]) == 1
    c.check_pointers()
    # nothing to do: no pointer is looked at
    for kw in (dict(tokens=0), dict(batch=0), dict(max_pages=0)):
        assert make(q8(**kw)).fn(ctypes.byref(q8(**kw)), *[None] * 10) == 0


def test_cache_overlaps():
    write().check_overlaps([3, 4, 5, 6], [1, 2, 7, 8, 9])
    read().check_overlaps([8, 9], range(1, 8))
    # rows of k and v interleaved in one buffer pass, overlapping ones do not
    c = read(q8(k_stride=1024, v_stride=1024))
    c.args[8] = A(7)
    for off, rc in ((504, 2), (520, 2)):  # (the second wraps into the next row)
        c.args[9] = ctypes.c_void_p(A(7).value + 2 * off)
        assert c() == rc and "overlap" in hb.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(window=-1), 2), (dict(sinks=-1), 2), (dict(page=16), 5), (dict(page=33), 5), (dict(sb=16), 5), (dict(sb=128), 5),
    (dict(max_pages=-1), 2), (dict(n_pages=0), 2), (dict(max_pages=1 << 25), 2)])
def test_step_sizes(kw, code):
    assert step(**kw)() == code and hb.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), 2), (dict(head_dim=32), 5), (dict(block=33), 5), (dict(block=0), 2), (dict(dtype=7), 4),
    (dict(flags=2), 2), (dict(flags=64), 2), (dict(n_q_heads=15), 2), (dict(n_q_heads=1 << 17, n_kv_heads=1 << 17), 5)])
def test_step_dims(kw, code):
    assert step(dims(**kw))() == code and hb.last_error()


def test_step_pointers():
    c = step()
    assert c.fn(None, *c.args[1:]) == 1
    for i in (1, 2, 3, 4, 5, 6, 7, 11, 13, 17):
        assert c(i, None) == 1, i
    for i in (1, 2, 3, 4, 5, 6, 7, 11, 13, 16, 17, 18):
        assert c(i, ODD) == 3, i
    need = hb.workspace_bytes(dims(), hb.OP_WINDOW_STEP_Q8, 168)
    big = step(max_pages=1000, window=60000)
    need = hb.workspace_bytes(dims(), hb.OP_WINDOW_STEP_Q8, 60068)
    assert need > 0 and big(18, None) == 6 and big(19, need - 1) == 6
    c = step(max_pages=1000, window=60000)
    c.check_overlaps([17, 18], [1, 2, 3, 4, 5, 6, 7, 11, 13, 16])
    assert step(dims(batch=0)).fn(ctypes.byref(dims(batch=0)), *step().args[1:]) == 0


def test_workspace_of_invalid_dims():
    assert hb.workspace_bytes(dims(head_dim=5), hb.OP_WINDOW_STEP_Q8, 100) == 0
    assert hb.workspace_bytes(dims(), hb.OP_WINDOW_STEP_Q8, -1) == 0
    assert hb.workspace_bytes(dims(), hb.OP_WINDOW_STEP_Q8, 2 ** 31 - 1) == 0


def test_binding_takes_device_tensors():
    k, p, s = torch.zeros(4, 2, 64), torch.zeros(3, 32, 2, 64).to(torch.float8_e4m3fn), torch.ones(3, 1, 2).to(torch.float8_e8m0fnu)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        hb.kv_pages_q8_write(k, k, p, p, s, s, i[None], i, i)
    with pytest.raises(TypeError):
        hb.kv_pages_q8_read(p, p, s, s, i[None], i, i, tokens=4)
    with pytest.raises(TypeError):
        hb.softmax_window_step_paged_q8(k[None], k[None], k[None], p, p, s, s, i[None], i, 5)


def packed(d=None, tokens=40, window=10, sinks=2, strides=(0, 0, 0)):
    # dims tokens window sinks q k v qs ks vs token_start out lse
    return Call("softmax_packed_prefill", [d or dims(), tokens, window, sinks] + [A(i) for i in range(3)] + list(strides)
                + [A(3), A(4), A(5), None], [4, 5, 6, 10, 11, 12], (12,))


def packed_gradient(d=None, tokens=40, window=10, sinks=2, strides=(0, 0, 0)):
    # dims tokens window sinks q k v qs ks vs token_start out lse dout dq dk dv ws bytes
    return Call("softmax_packed_backward", [d or dims(), tokens, window, sinks] + [A(i) for i in range(3)] + list(strides)
                + [A(3), A(4), A(5), A(6), A(7), A(8), A(9), A(10), 1 << 26, None],
                [4, 5, 6, 10, 11, 12, 13, 14, 15, 16])


@pytest.mark.parametrize("make", [packed, packed_gradient])
def test_packed_refusals(make):
    for kw, code in ((dict(tokens=-1), 2), (dict(tokens=(1 << 30) + 1), 2), (dict(window=-1), 2), (dict(sinks=-1), 2),
                     (dict(strides=(2040, 0, 0)), 2), (dict(strides=(0, 8, 0)), 2), (dict(strides=(0, 0, -512)), 2),
                     (dict(strides=(2052, 0, 0)), 3), (dict(strides=(0, 0, 1 << 25)), 2)):
        assert make(**kw)() == code and hb.last_error(), kw
    for kw, code in ((dict(batch=-1), 2), (dict(head_dim=32), 5), (dict(block=33), 5), (dict(dtype=7), 4), (dict(flags=2), 2),
                     (dict(n_q_heads=15), 2), (dict(n_q_heads=1 << 17, n_kv_heads=1 << 17), 5)):
        assert make(dims(**kw))() == code and hb.last_error(), kw
    assert make(dims(n_q_heads=65536, n_kv_heads=65536), tokens=1 << 30)() == 2  # the grid's limit
    c = make()
    assert c.fn(None, *c.args[1:]) == 1
    c.check_pointers()
    nothing = make(dims(batch=0))
    assert nothing() == 0 and make(tokens=0)() == 0


def test_packed_overlaps():
    packed().check_overlaps([11, 12], [4, 5, 6, 10])
    c = packed_gradient()
    c.check_overlaps([14, 15, 16, 17], [4, 5, 6, 10, 11, 12, 13])
    need = hb.workspace_bytes(dims(), hb.OP_PACKED_BACKWARD, 40)
    assert need > 0 and c(17, None) == 6 and c(18, need - 1) == 6 and c(17, ODD) == 3
    for bad in (dims(head_dim=5), dims(batch=0)):
        assert hb.workspace_bytes(bad, hb.OP_PACKED_BACKWARD, 100) == 0
    assert hb.workspace_bytes(dims(), hb.OP_PACKED_BACKWARD, 0) == 0
