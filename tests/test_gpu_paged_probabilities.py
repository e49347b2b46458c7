"""How many bits of its probabilities the paged attention multiplies with the values: O in fp32, so that its own rounding does not hide it,
against 64 bits, by norms.

Two bf16 terms: each rounding is off by 2^-8 of what it rounds at most, the two by 2^-16 of p.  They are independent of V, whose N(0, 1) columns
O sums with random signs, so that the norm of what they do to O is at most 2^-16 = 1.5e-5 of O's.  An fp32 exponent of up to 20 is off by
20 x 2^-24 = 1.2e-6, sums of 3000 terms by about 2^-24 x sqrt(3000) = 3.3e-6.  BAR is twice the sum.  One term: at most 2^-8 = 3.9e-3, and
as its errors are spread evenly over a step, whatever p is, a third of that or more."""
import numpy as np
import pytest
import torch

from paged_util import Batch, f64
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_paged_attention

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
BAR, ONE = 4e-5, 2.0 ** -8


def error(b, window=0, causal=True, **kw):
    O, _ = burst_paged_attention(b.q, *b.args(), window=window, causal=causal, out=torch.empty(b.q.shape, device="cuda"), **kw)
    want = b.reference(causal, window)[0]
    return np.linalg.norm(f64(O) - want) / np.linalg.norm(want)


@pytest.mark.parametrize("d", [128, 96, 64, 32])
@pytest.mark.parametrize("lengths", [[8, 23, 60, 2], [255, 256, 257, 200], [3000, 700]])
def test_single_tokens(d, lengths):
    b = Batch(lengths, [1] * len(lengths), 16, 4, d, seed=d)
    assert error(b, max_new=1) <= BAR


@pytest.mark.parametrize("d", [120, 104, 96, 80, 48, 32, 8])
@pytest.mark.parametrize("L,window", [(60, 0), (255, 0), (256, 0), (257, 0), (1500, 0), (1500, 255), (1500, 257)])
def test_chunks_of_other_widths(d, L, window):
    b = Batch([L, 40], [40, 1], 8, 2, d, seed=d + L)
    assert error(b, window) <= BAR


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("L,window,causal", [(60, 0, True), (255, 0, True), (256, 0, True), (1500, 0, False), (1500, 255, True)])
def test_chunks_on_request(d, L, window, causal):
    b = Batch([L, 40], [40, 1], 8, 2, d, seed=d + L)
    assert error(b, window, causal, full_p=True) <= BAR
    if causal:
        walk = PagedWalk(b.k_pages, b.v_pages, b.scale, window=window, full_p=True)
        O, lse = walk.step(b.q, b.k, b.v, b.table, b.lengths, b.starts)      # (the new tokens' keys are in the cache from here on)
        want = burst_paged_attention(b.q, *b.args(), window=window, full_p=True)
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("d", [128, 64])
def test_chunks_are_as_exact_with_few_keys_as_with_many(d):
    off = [error(Batch([L, L], [40, 30], 8, 2, d, seed=L)) for L in (100, 200, 254, 320, 600, 1500)]
    assert max(off) <= ONE and min(off) >= ONE / 4 and max(off) <= 1.25 * min(off), off
