"""What planning and keeping refuse, before any device call."""
import ctypes

import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_keep, burst_cache_plan
from test_paged_refusals import AT, E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, NULL, OK, paged, tensors


def plan(**kw):
    p = B.BurstPlan(**dict(dict(sequences=2, rows=3, pages=5, page=16, width=4, added=4096, lengths=4096, table=8192, free_pages=12288, free_count=16384, starts=20480,
                                totals=24576, slots=28672, positions=32768), **kw))
    return B.load().burst_cache_plan(ctypes.byref(p), NULL)


def test_plan():
    assert B.load().burst_cache_plan(None, NULL) == E_NULL
    for bad in (dict(sequences=-1), dict(sequences=4097), dict(rows=-1), dict(rows=1 << 20), dict(pages=-1), dict(width=-1), dict(page=8), dict(page=24), dict(page=0),
                dict(page=1 << 20, width=1 << 10), dict(table_stride=3), dict(table_stride=-4), dict(parents=4096, words=0), dict(parents=4096, words=1, most=-1),
                dict(parents=4096, words=1, most=5, parents_stride=4), dict(words=-1), dict(words=(1 << 20) + 1)):
        assert plan(**bad) == E_SHAPE, bad
    for name in ("added", "lengths", "table", "free_pages", "free_count", "starts", "totals", "slots", "positions"):
        assert plan(**{name: None}) == E_NULL, name
        assert plan(**{name: 4098 if name not in ("slots", "positions") else 4100}) == E_ALIGN, name
    assert plan(parents=4096, words=1, most=4) == E_NULL and plan(parents=4096, words=1, most=4, tree=4100) == E_ALIGN and plan(parents=4098, words=1, most=4, tree=4096) == E_ALIGN


def keep(p, pools=(4096, 8192), n=None, most=4, stride=0, kept=AT, counts=ctypes.c_void_p(8192), out=ctypes.c_void_p(12288)):
    at = None if pools is None else (ctypes.c_void_p * len(pools))(*pools)
    return B.load().burst_cache_keep(at, len(pools or ()) if n is None else n, kept, stride, most, counts, out, None if p is None else ctypes.byref(p), NULL)


def test_keep():
    assert keep(None) == E_NULL and keep(paged(dtype=5)) == E_DTYPE
    for bad in (dict(n=-1), dict(most=-1), dict(stride=3), dict(stride=-1), dict(pools=(4096, 4096)), dict(pools=(4096, 8192, 4096)), dict(out=AT), dict(out=ctypes.c_void_p(8192))):
        assert keep(paged(), **bad) == E_SHAPE, bad
    assert keep(paged(sequences=65536)) == E_SHAPE and keep(paged(page=8)) == E_SHAPE and keep(paged(page_strides=[0, 8, 64])) == E_SHAPE
    for bad in (dict(pools=None, n=2), dict(pools=(4096, None)), dict(kept=NULL), dict(counts=NULL), dict(out=NULL)):
        assert keep(paged(), **bad) == E_NULL, bad
    for bad in (dict(pools=(4096, 8193)), dict(kept=ctypes.c_void_p(4098)), dict(counts=ctypes.c_void_p(4098)), dict(out=ctypes.c_void_p(4098))):
        assert keep(paged(), **bad) == E_ALIGN, bad
    for name in ("starts", "lengths", "table"):
        assert keep(paged(**{name: None})) == E_NULL and keep(paged(**{name: 4098})) == E_ALIGN
    assert keep(paged(sequences=0), pools=None, n=2) == OK


def test_torch_calls():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)         # noqa: E731
    with pytest.raises(ValueError, match="table: device tensor"):
        burst_cache_plan(i(2), i(2), i(2, 4), i(5), i(1), 16, 3)
    t = tensors()
    with pytest.raises(ValueError, match="k_pages: device tensor"):
        burst_cache_keep(t["k_pages"], t["v_pages"], t["table"], t["lengths"], t["starts"], i(2, 3), i(2))
    with pytest.raises(ValueError, match="as many v_pages"):
        burst_cache_keep([t["k_pages"]] * 2, t["v_pages"], t["table"], t["lengths"], t["starts"], i(2, 3), i(2))
