"""Which kernel a paged attention runs, as its bits show: at d = 128 the kernel of longer chunks rounds P once, the one of single tokens does not."""
import numpy as np
import pytest
import torch

from paged_util import Batch, f64
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def attend(b, **kw):
    return burst_paged_attention(b.q, *b.args(), **kw)


@pytest.mark.parametrize("news", [[1, 1, 1, 1], [1, 0, 1, 1], [0, 4, 0, 0]])
def test_no_more_rows_than_sequences_are_single_tokens(news):
    """Nothing said about them; [0, 4, 0, 0] is no such batch, and right all the same."""
    b = Batch([300, 90, 700, 40], news, 16, 2, 128, seed=2)
    burst_cache_append(b.k, b.v, *b.args())                   # (what the step below does again)
    single, chunk = attend(b, max_new=1), attend(b, max_new=50)
    assert not torch.equal(single[0], chunk[0])
    for out in (attend(b), PagedWalk(b.k_pages, b.v_pages, b.scale).step(b.q, b.k, b.v, b.table, b.lengths, b.starts)):
        assert torch.equal(out[0], single[0]) and torch.equal(out[1], single[1])
        b.check(*out)
    more = Batch([300, 90, 700], [2, 1, 1], 16, 2, 128, seed=2)
    assert torch.equal(attend(more)[0], attend(more, max_new=50)[0])
    many = Batch([300, 90, 700], [1, 1, 1], 34, 2, 128, seed=2)          # 17 heads of a group: no kernel is made for them
    assert torch.equal(attend(many)[0], attend(many, max_new=50)[0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [128, 64, 96, 80, 32, 8])
@pytest.mark.parametrize("window", [0, 40])
def test_single_tokens_in_the_kernel_of_chunks(dtype, d, window):
    lengths = [1, 0, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 500, 1025]
    b = Batch(lengths, [1] * len(lengths), 4, 2, d, dtype=dtype, seed=d)
    b.check(*attend(b, max_new=100, window=window), window=window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_hidden_values_in_the_kernel_of_chunks(dtype, value):
    b = Batch([100, 203, 64], [1, 1, 1], 16, 2, 128, dtype=dtype, seed=4)
    for i, L in enumerate(b.lengths_list):
        last = int(b.table[i, (L - 1) // 16])
        if L % 16:
            b.k_pages[last, :, L % 16:] = value
            b.v_pages[last, :, L % 16:] = value
    for f in b.free:
        b.k_pages[f] = value
        b.v_pages[f] = value
    b.check(*attend(b, max_new=100))
    for p in (0, 3, 100):
        at = (int(b.table[1, p // 16]), slice(None), p % 16)
        b.k_pages[at], b.v_pages[at] = value, value
    b.check(*attend(b, max_new=100, window=60), window=60)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("d,H", [(128, 4), (64, 16), (96, 2)])
def test_rows_that_do_not_see_an_infinity_keep_their_bounds(dtype, value, where, d, H):
    """Keys 60 and 95 of 100 hold it, the new tokens are those from 55 on: whose window of five keys has neither is held to the bound of the same
    batch without them."""
    b = Batch([100, 64], [45, 1], H, 2, d, dtype=dtype, seed=5)
    O_ref, lse_ref, O_err, lse_err = b.reference(True, 5)
    pages = b.k_pages if where == "k" else b.v_pages
    for key in (60, 95):
        pages[int(b.table[0, key // 16]), :, key % 16] = value
    O, lse = attend(b, window=5, max_new=60)
    sees = np.array([any(p - 5 < key <= p for key in (60, 95)) for p in range(55, 100)] + [False])
    got, got_lse = f64(O), f64(lse)
    assert np.all(np.abs(got - O_ref)[~sees] <= O_err[~sees]) and np.all(np.abs(got_lse - lse_ref)[~sees] <= lse_err[~sees])
    assert sees.sum() == 10
    if where == "v":
        assert not np.isfinite(got[sees]).any() and np.all(np.abs(got_lse - lse_ref)[sees] <= lse_err[sees])
