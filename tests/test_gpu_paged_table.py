"""Sequences that have outgrown their row of the page table: tokens at positions from width x page on have no place in the cache.  They are
left out as tokens in pages that are none are, so that a table whose further entries are no pages is the reference."""
import numpy as np
import pytest
import torch

from paged_util import Batch, check_rotation, default_turns, f64
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def cut(b, width):
    """The batch with no pages from `width` on, and its table without those entries."""
    b.table[:, width:] = -1
    return b.k_pages, b.v_pages, b.table[:, :width], b.lengths, b.starts


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths,news", [([65, 40, 64], [1, 1, 1]), ([70, 64, 63], [9, 3, 2]), ([200, 90], [30, 90]), ([1000], [1])])
def test_appended_tokens_behind_the_table_are_left_out(dtype, lengths, news):
    b = Batch(lengths, news, 4, 2, 64, dtype=dtype, seed=len(news))
    args = cut(b, 4)                                          # 64 positions
    k0, v0 = b.k_pages.clone(), b.v_pages.clone()
    turns = default_turns(64)
    q = burst_cache_append(b.k, b.v, *args, q=b.q, turns=turns)
    pos = np.array([p for _, p in b.positions()])
    check_rotation("q", q, b.q, pos[:, None], f64(turns))     # (their queries have their own positions)
    for i, (s, p) in enumerate(b.positions()):
        if p < 64:
            at = (int(b.table[s, p // 16]), slice(None), p % 16)
            check_rotation("k", b.k_pages[at], b.k[i], np.array([p]), f64(turns))
            assert torch.equal(b.v_pages[at], b.v[i])
            k0[at], v0[at] = b.k_pages[at], b.v_pages[at]
    assert torch.equal(k0, b.k_pages) and torch.equal(v0, b.v_pages)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 30), (False, 0), (True, 1)])
@pytest.mark.parametrize("lengths,news", [([65, 40, 64], [1, 1, 1]), ([70, 64, 63], [9, 3, 2]), ([300, 90], [250, 90]), ([3000], [2990]), ([1000], [1])])
def test_tokens_behind_the_table_see_its_keys(dtype, causal, window, lengths, news):
    b = Batch(lengths, news, 8, 2, 64, dtype=dtype, seed=len(news))
    args = cut(b, 4)
    for max_new in (0, 1):
        O, lse = burst_paged_attention(b.q, *args, causal=causal, window=window, max_new=max_new)
        b.check(O, lse, causal, window)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_sequence_grows_out_of_its_table(dtype):
    """Single steps: what was in the cache stays as it was, and later tokens see it."""
    b = Batch([60], [1], 4, 2, 64, dtype=dtype)
    pages = b.k_pages, b.v_pages
    table = b.table[:, :4]
    walk = PagedWalk(*pages, 0.125, default_turns(64))
    for L in range(61, 72):
        before = [p.clone() for p in pages]
        b.lengths.fill_(L)
        O, lse = walk.step(b.q, b.k, b.v, table, b.lengths, b.starts, max_new=1)
        if L > 64:
            assert all(torch.equal(p, x) for p, x in zip(pages, before))
        else:
            assert not torch.equal(pages[0], before[0])
        assert torch.isfinite(O).all() and torch.isfinite(lse).all()


def test_lengths_beyond_every_position():
    """Lengths are cut to 2^30, and what they begin behind the table."""
    b = Batch([60, 20], [3, 1], 4, 2, 64)
    k0, v0 = b.k_pages.clone(), b.v_pages.clone()
    for L in ((1 << 30) - 1, 1 << 30, 0x7fffffff):
        b.lengths[0] = L
        burst_cache_append(b.k[:3], b.v[:3], *b.args()[:2], b.table[:1], b.lengths[:1], b.starts[:2])
        assert torch.equal(k0, b.k_pages) and torch.equal(v0, b.v_pages)
        for max_new in (0, 1):
            O, lse = burst_paged_attention(b.q[:3], *b.args()[:2], b.table[:1], b.lengths[:1], b.starts[:2], window=16, max_new=max_new)
            assert torch.isneginf(lse).all() and (O == 0).all()
            O, lse = burst_paged_attention(b.q[:3], *b.args()[:2], b.table[:1], b.lengths[:1], b.starts[:2], max_new=max_new)
            assert torch.isfinite(lse).all()
