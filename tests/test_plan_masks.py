"""Which plans a walk with a window takes: those with masks for it, or with branches that are shorter than either window."""
import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import CachePlan, burst_cache_plan
from test_cache_books_refusals import plan as c_plan
from test_paged_refusals import E_SHAPE


def a_plan(window=0, longest=None, words=1, trees=True):
    i = torch.zeros(3, dtype=torch.int64)
    p = CachePlan(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), i, i, torch.zeros(3, words, dtype=torch.int64) if trees else None)
    if trees:
        p.window, p.longest = window, longest
    return p


@pytest.mark.parametrize("plan,walk,longest,words,fits", [
    (0, 0, None, 1, True), (0, 64, None, 1, True), (0, 63, None, 1, False), (0, 64, None, 2, False), (0, 128, None, 2, True), (8, 8, None, 1, True), (8, 7, None, 1, False),
    (8, 0, None, 1, False), (64, 0, None, 1, True), (100, 500, None, 1, True), (0, 16, 16, 1, True), (0, 15, 16, 1, False), (15, 16, 16, 1, False), (16, 17, 16, 1, True)])
def test_masks_for(plan, walk, longest, words, fits):
    p = a_plan(plan, longest, words)
    assert p.masks_for(walk) == fits and a_plan(trees=False).masks_for(walk)
    pages = torch.zeros(2, 2, 16, 64)
    w = PagedWalk(pages, pages.clone(), 1.0, window=walk)
    t = [torch.zeros(3, h, 64) for h in (4, 2, 2)]
    with pytest.raises(ValueError, match="device tensor" if fits else "a plan with masks for a window"):   # (host tensors, which a step refuses next)
        w.planned_step(*t, torch.zeros(2, 1, dtype=torch.int32), p)


def test_a_plan_is_five_arrays():
    p = a_plan(3, 5)
    starts, lengths, slots, positions, tree = p
    assert len(p) == 5 and p[4] is tree is p.tree and p._fields == ("starts", "lengths", "slots", "positions", "tree")
    assert p._replace(tree=tree[:, :1]).window == 0           # (what other arrays are for is not known)


def test_windows_that_are_refused():
    assert c_plan(window=-1) == E_SHAPE and c_plan(window=-1, parents=4096, words=1, most=4, tree=4096) == E_SHAPE
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        burst_cache_plan(i, i, torch.zeros(2, 4, dtype=torch.int32), i, i[:1], 16, 3, torch.zeros(2, 3, dtype=torch.int32), 1, -1)


@pytest.mark.gpu
def test_negative_windows():
    i = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError, match="window"):
        burst_cache_plan(i, i.clone(), i.new_full((2, 4), -1), i.new_zeros(5), i.new_zeros(1), 16, 3, i.new_zeros(2, 3), 1, -1)
    with pytest.raises(B.BurstError):
        o, r = [i.new_empty(n) for n in (3, 2)], [torch.empty(3, dtype=torch.int64, device="cuda:0") for _ in range(2)]
        B.burst_cache_plan(i, i.clone(), i.new_full((2, 4), -1), i.new_zeros(5), i.new_zeros(1), 16, *o, *r, i.new_zeros(2, 3), r[0].new_empty(3, 1), -1)
