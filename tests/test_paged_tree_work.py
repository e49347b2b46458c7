"""The host's run of the integer logic of paged calls with trees, and what their entry points refuse."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_paged_attention
from test_paged_refusals import AT, E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, NULL, ODD, OK, paged, tensors

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_masks_ranges_and_units(tmp_path):
    exe = str(tmp_path / "driver")
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", os.path.join(ROOT, "paper_2403_09347_amd", "csrc"), os.path.join(ROOT, "tests", "paged_tree_driver.cpp"), "-o", exe]
    subprocess.run(cmd, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "tree checks failed: 0" in r.stdout, r.stdout[-3000:]


def attend(p, tree=AT, words=1, stride=0, ws=AT, size=1 << 40, **kw):
    a = dict(dict(Q=AT, K=AT, V=AT, O=AT, lse=AT), **kw)
    return B.load().burst_paged_tree_fwd(a["Q"], a["K"], a["V"], a["O"], a["lse"], tree, words, stride, ws, size, None if p is None else ctypes.byref(p), NULL)


def test_refusals():
    assert attend(None) == E_NULL and attend(paged(dtype=5)) == E_DTYPE
    for bad in (dict(words=0), dict(words=-1), dict(words=(1 << 20) + 1), dict(words=4, stride=3), dict(stride=-1)):
        assert attend(paged(), **bad) == E_SHAPE, bad
    assert attend(paged(causal=0)) == E_SHAPE and attend(paged(scale=0.0)) == E_SHAPE and attend(paged(page=8)) == E_SHAPE
    assert attend(paged(), tree=NULL) == E_NULL and attend(paged(), tree=ctypes.c_void_p(4100)) == E_ALIGN
    for name in ("Q", "K", "V", "O", "lse"):
        assert attend(paged(), **{name: NULL}) == E_NULL and attend(paged(), **{name: ODD}) == E_ALIGN, name
    need = B.burst_paged_workspace_bytes(paged())
    assert attend(paged(), ws=NULL) == E_NULL and attend(paged(), size=need - 1) == E_SHAPE
    assert attend(paged(rows=0), tree=NULL, Q=NULL) == attend(paged(sequences=0), tree=NULL, Q=NULL) == OK
    t = tensors()
    with pytest.raises(ValueError, match="k_pages: device tensor"):
        burst_paged_attention(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lengths"], t["starts"], tree=torch.zeros(3, 1, dtype=torch.int64))
