"""What the calls that normalise rows refuse, before any device call: the C entry points with bad blocks and pointers, and the torch calls with
tensors that do not fit."""
import ctypes

import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_append
from paper_2403_09347_amd.rotary import burst_norm_rotary, rotary_turns
from test_paged_refusals import AT, E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, NULL, OK, paged, rotary, rows, tensors


def norm_rows(frm=None, weight=0, from_strides=(0, 0, 0), **kw):
    t = B.BurstNormRows(rows=rows(**kw), from_=frm, weight=weight)
    t.from_strides[:] = from_strides
    return t


def weight(**kw):
    return B.BurstNormWeight(**dict(dict(w=4096), **kw))


def call(t, w=None, r=rotary(), n=1, weights=1, eps=1e-6, d=64, dtype=0):
    w = weight() if w is None else w
    return B.load().burst_norm_rotate(None if t is None else ctypes.byref(t), n, ctypes.byref(w), weights, eps, None if r is None else ctypes.byref(r), d, dtype, NULL)


def back(t, w=None, r=rotary(), n=1, weights=1, eps=1e-6, d=64, dtype=0, ws=AT, size=1 << 40):
    w = weight(dw=8192) if w is None else w
    return B.load().burst_norm_rotate_bwd(None if t is None else ctypes.byref(t), n, ctypes.byref(w), weights, eps, None if r is None else ctypes.byref(r), d, dtype,
                                          ws, size, NULL)


def test_blocks():
    for f, t in ((call, norm_rows), (back, lambda **kw: norm_rows(**dict(dict(frm=12288), **kw)))):
        assert f(None) == E_NULL and f(t(), r=rotary(turns=None)) == E_NULL
        for r in (dict(dims=0), dict(dims=66), dict(amplitude=float("nan")), dict(inverse=1)):
            assert f(t(), r=rotary(**r)) == E_SHAPE, r
        for eps in (0.0, -1.0, float("nan"), float("inf")):
            assert f(t(), eps=eps) == E_SHAPE, eps
        for bad in (dict(d=1), dict(d=129), dict(n=-1), dict(weights=-1), dict(weights=0)):
            assert f(t(), **dict(dict(r=None), **bad)) == E_SHAPE, bad
        assert f(t(), dtype=2) == E_DTYPE
        for bad in (dict(weight=1), dict(weight=-2), dict(B=-1), dict(heads=-1), dict(rows=-2), dict(rows=2 ** 31 - 255), dict(x_strides=[-64, 64, 64]),
                    dict(y_strides=[64, -1, 64]), dict(y_strides=[384, 64, 0]), dict(from_strides=[-1, 64, 64]), dict(positions=4096, positions_stride=-3),
                    dict(y=4096, y_strides=[1, 2, 64])):
            assert f(t(**bad)) == E_SHAPE, bad
        for bad in (dict(x=None), dict(B=1 << 20, heads=1 << 12, rows=1 << 12, x_strides=[0, 0, 64], y_strides=[1 << 24, 64, 1 << 18], x=None)):
            assert f(t(**bad)) == E_NULL, bad
        for bad in (dict(x=4097), dict(y=4097), dict(positions=4100)):
            assert f(t(**bad)) == E_ALIGN, bad
        assert f(t(), weight(w=None)) == E_NULL and f(t(), weight(w=4097)) == E_ALIGN and f(t(), weight(w=4098, f32=1)) == E_ALIGN
    assert call(norm_rows(y=None)) == E_NULL
    assert call(norm_rows(x_strides=[0, 0, 1], y_strides=[1 << 40, 1 << 20, 64], B=1 << 20, heads=1 << 12, rows=1 << 12)) == E_SHAPE   # 2^44 rows
    assert back(norm_rows()) == E_NULL and back(norm_rows(frm=12289)) == E_ALIGN and back(norm_rows(frm=12288), weight(dw=8193)) == E_ALIGN
    assert back(norm_rows(frm=8192, y=8192, from_strides=[1, 2, 64])) == E_SHAPE             # the gradient in the place of x, but elsewhere
    assert call(None, n=0) == OK and call(norm_rows(rows=0, x=None, y=None)) == OK and back(norm_rows(rows=0, x=None), weight()) == OK
    assert back(norm_rows(frm=12288, y=None), weight()) == OK                               # no gradient is wanted


def test_workspace():
    """A row of sums for every workgroup: 4 rows and all of the two heads each."""
    t, w = norm_rows(frm=12288, heads=2, rows=30), weight(dw=8192)
    size = lambda t, w, r=rotary(): B.load().burst_norm_workspace_bytes(ctypes.byref(t), 1, ctypes.byref(w), 1, 1e-6, ctypes.byref(r), 64, 0)   # noqa: E731
    need = size(t, w)
    assert need % (64 * 4) == 0 and 64 * 4 <= need <= 30 * 64 * 4
    assert back(t, w, size=need - 1) == E_SHAPE and back(t, w, ws=NULL) == E_NULL and back(t, w, ws=ctypes.c_void_p(4104)) == E_ALIGN
    assert size(t, weight()) == 0 and size(norm_rows(frm=12288, weight=1), w) == 0 and size(norm_rows(frm=12288, weight=-1), w) == 0


def store(p, how, r=None, **kw):
    a = dict(dict(K=AT, V=AT, Kp=AT, Vp=AT, Q=NULL, Qo=NULL), **kw)
    return B.load().burst_cache_store(a["K"], a["V"], a["Kp"], a["Vp"], a["Q"], a["Qo"], None if how is None else ctypes.byref(how),
                                      None if r is None else ctypes.byref(r), ctypes.byref(p), NULL)


def test_store():
    how = lambda **kw: B.BurstStore(**dict(dict(eps=1e-6), **kw))               # noqa: E731
    assert store(paged(), None) == E_NULL and store(paged(dtype=5), how()) == E_DTYPE
    for bad in (dict(eps=0.0, k_weight=4096), dict(eps=float("nan"), q_weight=4096), dict(positions=4096, offsets=4096)):
        assert store(paged(), how(**bad)) == E_SHAPE, bad
    assert store(paged(), how(), rotary(inverse=1)) == E_SHAPE and store(paged(), how(), rotary(dims=66)) == E_SHAPE
    for bad in (dict(slots=4100), dict(positions=4100), dict(offsets=4100), dict(k_weight=4097), dict(q_weight=4098, q_weight_f32=1)):
        assert store(paged(), how(**bad)) == E_ALIGN, bad
    for name in ("K", "V", "Kp", "Vp"):
        assert store(paged(), how(), **{name: NULL}) == E_NULL and store(paged(), how(), **{name: ctypes.c_void_p(4097)}) == E_ALIGN, name
    assert store(paged(), how(), Q=AT) == E_NULL
    for name in ("starts", "lengths", "table"):
        assert store(paged(**{name: None}), how(slots=4096)) == E_NULL and store(paged(**{name: 4098}), how(positions=4096)) == E_ALIGN
    assert store(paged(q_strides=[256, 64], o_strides=[512, 64]), how(), rotary(), Q=AT, Qo=AT) == E_SHAPE
    assert store(paged(rows=0), how(), K=NULL) == store(paged(sequences=0), how(slots=4096), K=NULL) == OK


def test_torch_calls():
    x, w, turns = torch.zeros(1, 2, 3, 64), torch.ones(64), rotary_turns(64, device="cpu")
    with pytest.raises(ValueError, match="tensors of bfloat16 or float32"):
        burst_norm_rotary(x, w, turns)
    with pytest.raises(ValueError, match="one entry of weights"):
        burst_norm_rotary([x, x], [w], turns)
    with pytest.raises(ValueError, match="one offset"):
        burst_norm_rotary([x, x], w, turns, offset=[1])
    with pytest.raises(ValueError, match="one offset"):
        burst_norm_rotary([], w, turns)
    t = tensors()
    with pytest.raises(ValueError, match="k_pages: device tensor"):
        burst_cache_append(t["k"], t["v"], t["k_pages"], t["v_pages"], t["table"], t["lengths"], t["starts"], k_norm=torch.ones(64))
