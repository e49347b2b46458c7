"""What the rotation and the paged calls refuse, before any device call: the C entry points with bad blocks and pointers, and the torch
calls with tensors that do not fit."""
import ctypes

import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention
from paper_2403_09347_amd.rotary import burst_rotary, rotary_turns

AT = ctypes.c_void_p(4096)                                    # never dereferenced
ODD = ctypes.c_void_p(4104)
NULL = ctypes.c_void_p(0)
OK, E_NULL, E_ALIGN, E_SHAPE, E_DTYPE = 0, -1, -2, -3, -4


def rotary(**kw):
    return B.BurstRotary(**dict(dict(turns=4096, dims=64, interleaved=0, amplitude=1.0, inverse=0), **kw))


def rows(**kw):
    strides = {k: kw.pop(k) for k in ("x_strides", "y_strides") if k in kw}
    t = B.BurstRows(**dict(dict(x=4096, y=8192, B=1, heads=2, rows=3), **kw))
    for k, v in strides.items():
        getattr(t, k)[:] = v
    return t


def rotate(t, r, n=1, d=64, dtype=0):
    return B.load().burst_rotate(None if t is None else ctypes.byref(t), n, None if r is None else ctypes.byref(r), d, dtype, NULL)


def test_rotate():
    r = rotary()
    assert rotate(rows(), None) == E_NULL and rotate(None, r) == E_NULL
    assert rotate(rows(), rotary(turns=None)) == E_NULL and rotate(rows(), rotary(turns=4100)) == E_ALIGN
    for bad in (dict(dims=0), dict(dims=63), dict(dims=66), dict(dims=-2), dict(amplitude=float("nan")), dict(amplitude=float("inf"))):
        assert rotate(rows(), rotary(**bad)) == E_SHAPE, bad
    for d in (1, 0, 129, -4):
        assert rotate(rows(), rotary(dims=2), d=d) == E_SHAPE
    assert rotate(rows(), r, dtype=2) == E_DTYPE and rotate(rows(), r, n=-1) == E_SHAPE
    assert rotate(rows(x=None), r) == E_NULL and rotate(rows(y=None), r) == E_NULL and rotate(rows(y=4097), r) == E_ALIGN
    assert rotate(rows(x=4098), r, dtype=1) == E_ALIGN and rotate(rows(positions=4100), r) == E_ALIGN
    for bad in (dict(B=-1), dict(heads=-1), dict(rows=-2), dict(x_strides=[-64, 64, 64]), dict(y_strides=[64, -1, 64]),
                dict(positions=4096, positions_stride=-3), dict(y=4096, y_strides=[1, 2, 64])):
        assert rotate(rows(**bad), r) == E_SHAPE, bad
    assert rotate(None, r, n=0) == OK and rotate(rows(rows=0, x=None, y=None), r) == OK


def paged(**kw):
    strides = {k: kw.pop(k) for k in ("page_strides", "q_strides", "kv_strides", "o_strides") if k in kw}
    p = B.BurstPagedParams(**dict(dict(sequences=2, rows=3, H=4, kv_heads=2, d=64, dtype=0, pages=5, page=16, width=4, causal=1, scale=0.125,
                                       starts=4096, lengths=4096, table=4096), **kw))
    for k, v in strides.items():
        getattr(p, k)[:] = v
    return p


def attend(p, ws=AT, size=1 << 40, **kw):
    a = dict(dict(Q=AT, K=AT, V=AT, O=AT, lse=AT), **kw)
    return B.load().burst_paged_fwd(a["Q"], a["K"], a["V"], a["O"], a["lse"], ws, size, None if p is None else ctypes.byref(p), NULL)


def append(p, r=None, offsets=NULL, **kw):
    a = dict(dict(K=AT, V=AT, Kp=AT, Vp=AT, Q=NULL, Qo=NULL), **kw)
    return B.load().burst_cache_append(a["K"], a["V"], a["Kp"], a["Vp"], a["Q"], a["Qo"], offsets, None if r is None else ctypes.byref(r),
                                       None if p is None else ctypes.byref(p), NULL)


def test_blocks_of_paged_calls():
    assert attend(None) == append(None) == E_NULL
    assert attend(paged(dtype=5)) == append(paged(dtype=5)) == E_DTYPE
    for bad in (dict(sequences=-1), dict(sequences=1 << 30), dict(rows=-1), dict(rows=1 << 30), dict(max_new=-1), dict(pages=-1), dict(width=-1),
                dict(window=-1), dict(d=0), dict(d=136), dict(d=60), dict(d=66, dtype=1), dict(H=0), dict(H=5), dict(kv_heads=0), dict(page=8),
                dict(page=48), dict(page=0), dict(page=1 << 20, width=1 << 10), dict(table_stride=3), dict(page_strides=[8, 8, 56]),
                dict(page_strides=[-8, 8, 64]), dict(page_strides=[64, 64, 1 << 25]), dict(q_strides=[-64, 64]), dict(kv_strides=[64, -64]),
                dict(o_strides=[-1, 64])):
        assert attend(paged(**bad)) == append(paged(**bad)) == E_SHAPE, bad
        assert B.burst_paged_workspace_bytes(paged(**bad)) == 0
    for bad in (dict(rows=(1 << 30) - 1, H=4096, kv_heads=4096), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_strides=[260, 64]), dict(o_strides=[256, 60]),
                dict(page_strides=[2048, 1024, 68])):
        assert attend(paged(**bad)) == E_SHAPE, bad
    assert attend(paged(sequences=0), Q=NULL) == attend(paged(rows=0), Q=NULL) == append(paged(sequences=0), K=NULL) == append(paged(rows=0), K=NULL) == OK


def test_pointers_of_paged_calls():
    for name in ("Q", "K", "V", "O", "lse"):
        assert attend(paged(), **{name: NULL}) == E_NULL, name
        assert attend(paged(), **{name: ODD}) == E_ALIGN, name
    for name in ("starts", "lengths", "table"):
        assert attend(paged(**{name: None})) == append(paged(**{name: None})) == E_NULL
        assert attend(paged(**{name: 4098})) == append(paged(**{name: 4098})) == E_ALIGN
    need = B.burst_paged_workspace_bytes(paged())
    assert need > 0 and attend(paged(), ws=NULL) == E_NULL and attend(paged(), ws=ODD) == E_ALIGN and attend(paged(), size=need - 1) == E_SHAPE
    for name in ("K", "V", "Kp", "Vp"):
        assert append(paged(), **{name: NULL}) == E_NULL, name
        assert append(paged(), **{name: ctypes.c_void_p(4097)}) == E_ALIGN, name
    assert append(paged(), Q=AT) == E_NULL and append(paged(), offsets=ctypes.c_void_p(4100)) == E_ALIGN
    assert append(paged(), rotary(turns=None)) == E_NULL and append(paged(), rotary(dims=66)) == E_SHAPE
    assert append(paged(q_strides=[256, 64], o_strides=[512, 64]), rotary(), Q=AT, Qo=AT) == E_SHAPE      # in place, but elsewhere


def test_workspace_sizes():
    """Two partial results of 16 (128) rows and their statistics for every run: at most 1024 and 512 runs, fewer where there is less work.
    The arrays on the device have no part in it; 32 bytes a run for what is to be joined."""
    one = 2 * 16 * (64 + 2) * 4 + 32
    assert B.burst_paged_workspace_bytes(paged(sequences=64, rows=64, width=100, max_new=1)) == 1024 * one
    assert B.burst_paged_workspace_bytes(paged(sequences=64, rows=64, width=100)) == 512 * (8 * (one - 32) + 32)
    assert B.burst_paged_workspace_bytes(paged(sequences=1, rows=1, H=1, kv_heads=1, width=1, max_new=1)) < 64 * one
    assert B.burst_paged_workspace_bytes(paged(starts=None, lengths=None, table=None)) > 0


def tensors(S=2, T=3, H=4, KV=2, d=64, pages=5, page=16, width=4, dtype=torch.bfloat16):
    z = lambda *s: torch.zeros(*s, dtype=dtype)               # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)         # noqa: E731
    return dict(q=z(T, H, d), k=z(T, KV, d), v=z(T, KV, d), k_pages=z(pages, KV, page, d), v_pages=z(pages, KV, page, d), table=i(S, width),
                lengths=i(S), starts=i(S + 1))


def test_torch_calls_refuse_host_tensors_and_lists_that_do_not_fit():
    t = tensors()
    cache = [t[n] for n in ("k_pages", "v_pages", "table", "lengths", "starts")]
    with pytest.raises(ValueError, match="k_pages: device tensor"):
        burst_paged_attention(t["q"], *cache)
    with pytest.raises(ValueError, match="k_pages: device tensor"):
        burst_cache_append(t["k"], t["v"], *cache)
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError, match="tensors of bfloat16 or float32"):
        burst_rotary(x, rotary_turns(64, device="cpu"))
    with pytest.raises(ValueError, match="one offset"):
        burst_rotary([x, x], rotary_turns(64, device="cpu"), offset=[1])
    with pytest.raises(ValueError, match="one offset"):
        burst_rotary([], rotary_turns(64, device="cpu"))
    for bad in (dict(dims=3), dict(dims=0), dict(dims=8, base=0.0), dict(dims=8, factor=-1.0), dict(dims=8, scaling="other")):
        with pytest.raises(ValueError):
            rotary_turns(**bad, device="cpu")


def test_sizes_of_rotated_tensors():
    """Up to 2^31 - 256: the rows and heads of a workgroup are counted past the last one in 32 bits."""
    for size in ("B", "heads", "rows"):
        for n in (0x7fffff01, 0x7fffffff):
            assert rotate(rows(**{size: n}), rotary()) == E_SHAPE, (size, n)


def test_rows_that_would_be_written_to_one_place():
    for size, strides in (("B", [0, 640, 64]), ("heads", [640, 0, 64]), ("rows", [640, 64, 0])):
        assert rotate(rows(**dict(dict(B=1, heads=1, rows=1), **{size: 2}), y_strides=strides), rotary()) == E_SHAPE, size
    for strides in ([0, 64], [256, 0]):
        assert attend(paged(o_strides=strides)) == append(paged(o_strides=strides)) == E_SHAPE, strides
    for strides in ([0, 1024, 64], [2048, 0, 64]):
        assert append(paged(page_strides=strides)) == E_SHAPE, strides
