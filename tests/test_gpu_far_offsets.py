"""Rows behind the first 2^31 elements of a tensor: norms with their gradients, storing, trees and keeping in a pool of pages that large."""
import numpy as np
import pytest
import torch

import norm_util as nu
from paged_util import default_turns, f64
from paper_2403_09347_amd.paged import burst_cache_append, burst_cache_keep
from paper_2403_09347_amd.rotary import burst_norm_rotary
from test_gpu_cache_store import check as check_store, places, weight
from test_gpu_paged_tree import check as check_tree
from tree_util import TreeBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def test_norms():
    d, N = 128, (1 << 24) + 3
    x = torch.zeros(1, 1, N, d, dtype=BF16, device=DEV)
    g = torch.zeros(1, 1, N, d, dtype=BF16, device=DEV)
    assert x.numel() > 1 << 31
    ends = [slice(0, 20), slice(N - 40, N)]                    # (rows between them are zeros: their terms of dw as well)
    for at in ends:
        x[:, :, at] = torch.randn(x[:, :, at].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(BF16)
        g[:, :, at] = torch.randn(x[:, :, at].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(2)).to(BF16)
    x.requires_grad_(True)
    w, turns = weight(d, torch.float32, 3).requires_grad_(True), default_turns(d)
    y = burst_norm_rotary(x, w, turns, 1e-5)
    dx, dw = torch.autograd.grad(y, [x, w], g)
    parts = []
    for at in ends:
        how = dict(pos=np.arange(at.start, at.stop)[None, None], turns=f64(turns))
        nu.check_forward("y", y[:, :, at], x[:, :, at], w, 1e-5, **how)
        nu.check_dx("dx", dx[:, :, at], x[:, :, at], w, g[:, :, at], 1e-5, **how)
        parts.append(nu.dw_terms(x[:, :, at], w, g[:, :, at], 1e-5, **how))
    nu.check_dw("dw", dw, parts)
    assert not bool(y[:, :, 20:N - 40].any()) and not bool(dx[:, :, 20:N - 40].any())


def test_pages():
    b = TreeBatch([300, 77], [20, 33], 4, 1, 128, seed=3)
    n, pages = b.k_pages.shape[0], (1 << 20) + 40
    pools = []
    for small in (b.k_pages, b.v_pages):
        pool = torch.zeros(pages, 1, 16, 128, dtype=BF16, device=DEV)
        assert pool.numel() > 1 << 31
        pool[-n:] = small
        pools.append(pool)
    b.k_pages, b.v_pages = pools
    b.table = torch.where(b.table >= 0, b.table + (pages - n), b.table)
    check_tree(b, name="attention")
    slots, pos = places(b)
    turns, wk = default_turns(128), weight(128, BF16, 2)
    before = [p[-n:].clone() for p in pools]
    burst_cache_append(b.k, b.v, *b.args(), turns=turns, k_norm=wk, eps=1e-6, slots=slots, positions=pos)
    far = slots - (pages - n) * 16
    b.k_pages, b.v_pages = (p[-n:] for p in pools)
    check_store(b, before, None, far, pos, None, wk, turns)
    before = [p.clone() for p in (b.k_pages, b.v_pages)]
    kept = torch.tensor([[0, 5, 9], [2, 3, 30]], dtype=torch.int32, device=DEV)
    counts = torch.tensor([3, 3], dtype=torch.int32, device=DEV)
    burst_cache_keep(pools[0], pools[1], b.table, b.lengths, b.starts, kept, counts)
    for pool, old in zip((b.k_pages, b.v_pages), before):
        first = 0
        for s, m in enumerate(b.news):
            for j, k in enumerate(kept[s].tolist()):
                f, t = int(far[first + k]), int(far[first + j])
                assert torch.equal(pool[t // 16, :, t % 16], old[f // 16, :, f % 16])
            first += m
