"""Refusals of the norm and rotation, the page plan and the windowed softmax:
every check runs on the host before anything is enqueued (the pointers are
small fake addresses that no kernel may see)."""
import ctypes

import pytest
import torch

from paper_2608_06628_amd import binding as hb


def A(i):
    return ctypes.c_void_p(0x10000000 * (i + 1))  # 256 MiB apart, never dereferenced


ODD = ctypes.c_void_p(0x1008)


def dims(**kw):
    base = dict(batch=2, n_q_heads=16, n_kv_heads=4, head_dim=128, block=32, feat_dim=64, dtype=hb.HYB_BF16, n_slots=1,
                flags=0)
    base.update(kw)
    return hb.Dims(*[base[n] for n, _ in hb.Dims._fields_])


def rope(**kw):
    base = dict(tokens=8, n_q_heads=4, n_kv_heads=2, head_dim=128, rot_dim=128, layout=0, dtype=hb.HYB_BF16,
                grad_dtype=hb.HYB_F32, flags=0, eps=1e-6, rot_scale=1.0, q_stride=0, k_stride=0, v_stride=0,
                q_out_stride=0, k_out_stride=0)
    base.update(kw)
    return hb.RopeDims(*[base[n] for n, _ in hb.RopeDims._fields_])


class Call:
    """A call that passes its checks up to the launch, of which one argument is
    changed at a time."""

    def __init__(self, fn, args, ptrs, optional=()):
        self.fn, self.args, self.ptrs, self.optional = getattr(hb.load(), fn), args, ptrs, optional
        self.odd = {}

    def __call__(self, at=None, value=None):
        args = list(self.args)
        if at is not None:
            args[at] = value
        return self.fn(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args])

    def check_pointers(self):
        for i in self.ptrs:
            if i not in self.optional:
                assert self(i, None) == 1, i
                assert "NULL" in hb.last_error() or "required" in hb.last_error()
            assert self(i, self.odd.get(i, ODD)) == 3, i

    def check_overlaps(self, written, read):
        for w in written:
            for r in list(read) + [x for x in written if x != w]:
                assert self(w, self.args[r]) == 2, (w, r)
                assert "overlap" in hb.last_error()


def forward(d=None):
    return Call("hybrid_qk_norm_rope", [d or rope()] + [A(i) for i in range(8)] + [None], range(1, 9), (3, 4))


def paged(d=None, n_pages=4, page=32):
    # dims q k v wq wk positions inv_freq slots q_out k_out k_pages v_pages
    return Call("hybrid_qk_norm_rope_paged", [d or rope()] + [A(i) for i in range(12)] + [n_pages, page, None],
                range(1, 13), (4, 5, 10))


def gradient(d=None):
    # dims q k wq wk positions inv_freq dq_out dk_out dq dk dwq dwk ws bytes
    return Call("hybrid_qk_norm_rope_backward", [d or rope()] + [A(i) for i in range(13)] + [1 << 20, None],
                range(1, 14))


@pytest.mark.parametrize("make", [forward, paged, gradient])
@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), 2), (dict(n_q_heads=0), 2), (dict(n_kv_heads=0), 2), (dict(head_dim=96), 5), (dict(rot_dim=4), 5),
    (dict(rot_dim=136), 5), (dict(rot_dim=-8), 5), (dict(layout=2), 2), (dict(dtype=3), 4), (dict(grad_dtype=-1), 4),
    (dict(flags=2), 2), (dict(eps=0.0), 2), (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2),
    (dict(rot_scale=float("inf")), 2), (dict(q_stride=504), 2), (dict(k_stride=8), 2), (dict(q_stride=516), 3),
    (dict(q_stride=-512), 2), (dict(k_out_stride=248), 2), (dict(v_stride=1 << 40), 2)])
def test_rope_dims(make, kw, code):
    assert make(rope(**kw))() == code and hb.last_error()
    assert hb.load().hybrid_rope_workspace_bytes(ctypes.byref(rope(**kw))) == 0


def test_rope_pointers():
    for make in (forward, paged, gradient):
        c = make()
        assert c.fn(None, *c.args[1:]) == 1
    forward().check_pointers()
    paged().check_pointers()
    c = gradient()
    for i in (1, 2, 5, 6, 7, 8, 9, 10):
        assert c(i, None) == 1, i
    for i in range(1, 14):
        assert c(i, ODD) == 3, i
    # the weights' gradients where, and only where, there are weights
    for i in (3, 4, 11, 12):
        assert c(i, None) == 1 and "dwq" in hb.last_error()
    assert c(13, None) == 6 and c(14, 0) == 6
    assert c(14, hb.load().hybrid_rope_workspace_bytes(ctypes.byref(rope())) - 1) == 6


def test_rope_overlaps():
    forward().check_overlaps([7, 8], range(1, 7))
    paged().check_overlaps([9, 10, 11, 12], range(1, 9))
    gradient().check_overlaps([9, 10, 11, 12, 13], [1, 2, 3, 4, 5, 6, 7, 8])
    # outputs in one buffer: side by side passes (to the next refusal), overlapping does not
    d = rope(q_out_stride=768, k_out_stride=768)
    c = forward(d)
    c.args[7] = A(6)
    c.args[8] = ctypes.c_void_p(A(6).value + 2 * 504)
    assert c() == 2 and "overlap" in hb.last_error()
    c.args[8] = ctypes.c_void_p(A(6).value + 2 * 520)
    assert c() == 2 and "overlap" in hb.last_error()  # wraps into the next row


def test_rope_pages():
    assert paged(n_pages=0)() == 2 and paged(page=0)() == 2


def test_rope_nothing_to_do():
    lib = hb.load()
    d = ctypes.byref(rope(tokens=0))
    assert lib.hybrid_qk_norm_rope(d, *[None] * 9) == 0
    assert lib.hybrid_qk_norm_rope_paged(d, *[None] * 12, 1, 1, None) == 0
    assert lib.hybrid_qk_norm_rope_backward(d, *[None] * 13, 0, None) == 0


def plan(**kw):
    base = dict(batch=4, max_pages=8, page=32, n_free=10, max_tokens=64)
    base.update(kw)
    return Call("kv_pages_plan", list(base.values()) + [A(i) for i in range(8)] + [None], range(5, 13))


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), 2), (dict(batch=4097), 5), (dict(max_pages=-1), 2), (dict(page=0), 5), (dict(page=48), 5),
    (dict(page=1 << 17), 5), (dict(n_free=-1), 2), (dict(max_tokens=-1), 2), (dict(max_pages=1 << 26), 2)])
def test_plan_sizes(kw, code):
    assert plan(**kw)() == code and hb.last_error()


def test_plan_pointers_and_overlaps():
    c = plan()
    c.odd[7] = ctypes.c_void_p(0x1002)  # free_pages: a list's place of 4 bytes
    c.check_pointers()
    # prefix_len new_len free_pages | page_table slots positions token_start counts
    plan().check_overlaps([8, 9, 10, 11, 12], [5, 6, 7])
    assert hb.load().kv_pages_plan(0, 0, 32, 0, 0, *[None] * 9) == 0


def step(d=None, window=64, sinks=4, need=1 << 24):
    # dims q k v k_pages v_pages n_pages page_size table max_pages prefix window sinks block_len out ws bytes
    return Call("softmax_window_step_paged",
                [d or dims(), A(0), A(1), A(2), A(3), A(4), 16, 64, A(5), 8, A(6), window, sinks, A(7), A(8), A(9), need,
                 None], (1, 2, 3, 4, 5, 8, 10, 13, 14, 15), (13, 15))


def test_window_step():
    assert step(window=-1)() == 2 and step(sinks=-1)() == 2
    assert step(dims(n_kv_heads=1))() == 5 and "softmax_window_step_paged" in hb.last_error()
    assert step(dims(block=33))() == 5 and step(dims(flags=2))() == 2 and step(dims(dtype=5))() == 4
    c = step()
    c.check_pointers()
    c.check_overlaps([14], [1, 2, 3, 4, 5, 8, 10, 13])
    for at, v, code in ((6, 0, 2), (7, 48, 5), (7, 16, 5), (9, -1, 2), (9, 1 << 26, 2)):
        assert c(at, v) == code
    # a long cache needs a workspace by what is seen of it, not by its length
    lib = hb.load()
    big = [a for a in step(window=2048).args]
    big[9] = 1024
    need = lib.hybrid_workspace_bytes(ctypes.byref(dims()), hb.OP_WINDOW_STEP, 2048 + 4 + 64)
    assert 0 < need < lib.hybrid_workspace_bytes(ctypes.byref(dims()), hb.OP_WINDOW_STEP, 65536)
    big[16] = need - 1
    c = Call("softmax_window_step_paged", big, ())
    assert c() == 6 and c(15, None) == 6
    for at in (1, 2, 3, 4, 5, 8, 10, 13):  # the workspace over an input
        d = Call("softmax_window_step_paged", big, ())
        d.args[16] = need
        assert d(15, d.args[at]) == 2 and "overlap" in hb.last_error()
    assert lib.softmax_window_step_paged(ctypes.byref(dims(batch=0)), *[None] * 5, 0, 64, None, 0, None, 0, 0, None, None,
                                         None, 0, None) == 0


def prefill(d=None, T=100, window=64, sinks=4):
    return Call("softmax_window_prefill", [d or dims(), T, window, sinks] + [A(i) for i in range(7)] + [1 << 24, None],
                range(4, 11), (7, 9, 10))


def backward(d=None, T=100, window=64, sinks=4):
    # q k v seq_lens out lse dout dq dk dv ws
    return Call("softmax_window_backward", [d or dims(), T, window, sinks] + [A(i) for i in range(11)] + [1 << 30, None],
                range(4, 14), (7,))


@pytest.mark.parametrize("make", [prefill, backward])
def test_window_sizes(make):
    for T in (0, -1, (1 << 30) + 1):
        assert make(T=T)() == 2
    assert make(window=-1)() == 2 and make(sinks=-1)() == 2
    for kw, code in ((dict(head_dim=96), 5), (dict(block=33), 5), (dict(block=0), 2), (dict(n_kv_heads=3), 2),
                     (dict(dtype=9), 4), (dict(flags=4), 2), (dict(flags=16), 2), (dict(batch=-1), 2)):
        assert make(dims(**kw))() == code, kw
    assert make(dims(batch=1 << 20), T=1 << 20)() == 2  # more workgroups than a grid has
    make().check_pointers()


def test_window_overlaps():
    prefill().check_overlaps([8, 9], [4, 5, 6, 7])
    backward().check_overlaps([11, 12, 13], [4, 5, 6, 7, 8, 9, 10])
    lib = hb.load()
    need = lib.hybrid_workspace_bytes(ctypes.byref(dims()), hb.OP_WINDOW_BACKWARD, 100)
    c = backward()
    assert need > 0 and c(15, need - 1) == 6 and c(14, None) == 6 and c(14, ODD) == 3
    for at in (4, 9, 11):
        assert c(14, c.args[at]) == 2
    z = ctypes.byref(dims(batch=0))
    assert lib.softmax_window_prefill(z, 10, 0, 0, *[None] * 7, 0, None) == 0
    assert lib.softmax_window_backward(z, 10, 0, 0, *[None] * 11, 0, None) == 0


def test_binding_takes_device_tensors_only():
    t = torch.zeros(4, 2, 64)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: hb.hybrid_qk_norm_rope(t, t, None, i), lambda: hb.kv_pages_plan(i, i, i.view(2, 2), i, 32, 4),
                 lambda: hb.softmax_window_prefill(t[None], t[None], t[None], 1, 1)):
        with pytest.raises(TypeError):
            call()


def test_workspace_of_nothing():
    """Sizes of empty calls are 0, for every op, and no query ends the process."""
    lib = hb.load()
    for op in (hb.OP_WINDOW_STEP, hb.OP_WINDOW_PREFILL, hb.OP_WINDOW_BACKWARD):
        for d, extent in ((dims(batch=0), 100), (dims(), -1), (dims(head_dim=7), 10), (dims(batch=0), 0)):
            assert lib.hybrid_workspace_bytes(ctypes.byref(d), op, extent) == 0
        lib.hybrid_workspace_bytes(ctypes.byref(dims()), op, 2 ** 31 - 1)
    assert lib.hybrid_workspace_bytes(ctypes.byref(dims()), hb.OP_WINDOW_BACKWARD, 0) == 0
    assert lib.hybrid_rope_workspace_bytes(ctypes.byref(rope(tokens=0))) == 0
    assert lib.hybrid_rope_workspace_bytes(None) == 0


def test_too_many_heads():
    d = dims(n_q_heads=1 << 17, n_kv_heads=1 << 17, batch=1)
    for make in (prefill, backward, step):
        assert make(d)() == 5 and "heads" in hb.last_error()


def test_more_workgroups_than_a_grid_holds():
    d = dims(batch=1 << 24, n_q_heads=1, n_kv_heads=1)
    for make in (prefill, backward):
        assert make(d, T=1)() != 0 and "grid limit" in hb.last_error()
    d = dims(batch=2 ** 31 - 1, n_q_heads=65536, n_kv_heads=65536)
    for make in (prefill, backward):
        assert make(d, T=1 << 30)() != 0 and "grid limit" in hb.last_error()


def test_rows_of_a_tensor():
    """Row strides as the library takes them: an expanded tensor has none."""
    t = torch.zeros(6, 4, 64)
    rows = lambda x: hb._rows(-1, x, "q", torch.float32, x.shape)[1]
    assert rows(t) == 256 and rows(t[::2]) == 512 and rows(t[:1]) == 0 and rows(t[:0]) == 0
    assert rows(t[:, :1]) == 256 and rows(t[:1].expand(1, 4, 64)) == 0
    for bad in (t[:1].expand(6, 4, 64), t[:, :, ::2], t[:, ::2], t[:, :1].expand(6, 4, 64), t.transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            rows(bad)
