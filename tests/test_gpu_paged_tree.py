"""Attention of trees of drafted tokens over a paged cache, against 64 bits."""
import random

import numpy as np
import pytest
import torch

from paged_util import Batch, f64
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_paged_attention
from tree_util import TreeBatch, as_words, random_parents, tree_mask

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def run(b, window=0, **kw):
    O, lse = burst_paged_attention(b.q, *b.args(), scale=b.scale, window=window, tree=b.tree, **kw)
    torch.cuda.synchronize()
    return O, lse


def check(b, window=0, name="", **kw):
    O, lse = run(b, window, **kw)
    b.check(O, lse, window=window, name=name)
    return O, lse


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [8, 32, 64, 80, 96, 104, 128])
@pytest.mark.parametrize("H,KV", [(2, 2), (8, 2), (3, 1), (17, 1)])
def test_kernels(dtype, d, H, KV):
    """Few rows a sequence (the short kernel; max_new tells it), and more."""
    for lengths, news, most in (([40, 5, 130, 3], [4, 4, 2, 3], 4), ([70, 300, 5, 129], [40, 64, 5, 1], 0)):
        b = TreeBatch(lengths, news, H, KV, d, dtype=dtype, seed=d + H, spare_rows=2)
        check(b, max_new=most, name=f"{lengths}")


@pytest.mark.parametrize("words,news", [(1, [64, 63, 1, 0, 33]), (2, [128, 65, 64, 100, 7]), (4, [256, 200, 129, 3, 255])])
@pytest.mark.parametrize("base", [0, 1, 15, 16, 63, 64, 100])
def test_sizes_and_where_trees_begin(words, news, base):
    """Trees that begin at any place of a tile and end in any, of as many tokens as a mask has bits; bits beyond a tree mean nothing."""
    b = TreeBatch([base + 3 * i + n for i, n in enumerate(news)], news, 4, 2, 64, words=words, seed=base, junk=True, pool="seq")
    check(b)


@pytest.mark.parametrize("dtype,group", [(BF16, 1), (BF16, 4), (F32, 2)])
@pytest.mark.parametrize("window", [1, 2, 7, 40, 1000])
def test_windows(dtype, group, window):
    for news in ([5, 60, 130, 16], [3, 4, 1, 2]):
        b = TreeBatch([5 + 7, 60 + 300, 130 + 90, 16 + 2000], news, 2 * group, 2, 64, dtype=dtype, words=2, seed=window, junk=True)
        check(b, window, max_new=max(news))


def test_any_masks():
    """Masks that are no trees: nothing at all, everything, later tokens, not the token itself; a sequence that has nothing before."""
    rng = random.Random(3)
    for lengths, news in (([40, 70, 64, 200], [40, 64, 30, 64]), ([4, 12, 3, 64], [4, 4, 3, 2])):
        masks = [[rng.choice([0, (1 << n) - 1, rng.getrandbits(n), 1 << rng.randrange(n), (1 << n) - 1 - (1 << t)]) for t in range(n)] for n in news]
        masks[0][1] = 0
        b = TreeBatch(lengths, news, 4, 2, 64, masks=masks, seed=9)
        O, lse = check(b, max_new=max(news))
        assert bool((O[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
        check(b, 5, max_new=max(news))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunks_of_prompts_beside_trees(dtype):
    """More new tokens than bits: as without masks."""
    news = [100, 12, 65, 300, 64]
    b = TreeBatch([100, 500, 700, 310, 64], news, 8, 2, 64, dtype=dtype, seed=2)
    for window in (0, 50):
        O, lse = check(b, window)
        plain = Batch([100, 500, 700, 310, 64], news, 8, 2, 64, dtype=dtype, seed=2)
        want = burst_paged_attention(plain.q, *plain.args(), scale=plain.scale, window=window)
        for first, n in ((0, 100), (112, 65), (177, 300)):
            assert torch.allclose(O[first:first + n].float(), want[0][first:first + n].float(), atol=2e-2 if dtype == BF16 else 2e-5, rtol=0)
            assert torch.allclose(lse[first:first + n], want[1][first:first + n], atol=1e-4, rtol=0)


@pytest.mark.parametrize("group", [1, 4])
def test_a_chain_is_causal(group):
    news = [64, 5, 1, 33]
    masks = [[(2 << t) - 1 for t in range(n)] for n in news]
    b = TreeBatch([64, 300, 17, 1000], news, 2 * group, 2, 128, masks=masks, seed=4)
    O, lse = check(b)
    b2 = Batch([64, 300, 17, 1000], news, 2 * group, 2, 128, seed=4)
    b2.check(O, lse, name="causal")


@pytest.mark.parametrize("news", [[4, 3], [50, 64]])
def test_hidden_keys_hold_anything(news):
    """Infinities and NaN in keys and values that a row does not see: other branches, the page's rows behind the sequence, pages that are none."""
    lengths = [200 + news[0], 64 + news[1]]
    b = TreeBatch(lengths, news, 8, 2, 64, seed=6, spare_pages=2)
    n, L = news[0], lengths[0]
    lone = n - 2                                              # a token that nothing but itself sees
    b.masks[0] = [m & ~(1 << lone) for m in b.masks[0]]
    b.masks[0][lone] |= 1 << lone
    b.tree[:n] = torch.from_numpy(as_words(b.masks[0], 1)).to(DEV)
    at = lambda s, p: (int(b.table[s, p // 16]), p % 16)     # noqa: E731
    want = run(b, max_new=max(news))
    page, row = at(0, L - n + lone)
    b.k_pages[page, :, row], b.v_pages[page, :, row] = float("nan"), float("inf")
    for s in (0, 1):                                          # behind the ends
        for p in range(lengths[s], -(-lengths[s] // 16) * 16):
            page, row = at(s, p)
            b.k_pages[page, :, row], b.v_pages[page, :, row] = float("inf"), float("nan")
    O, lse = run(b, max_new=max(news))
    others = [t for t in range(sum(news)) if t != lone]
    O_ref, lse_ref, O_err, lse_err = TreeBatch.reference(TreeBatchWithout(b, lone))
    got, got_lse = f64(O)[others], f64(lse)[others]
    assert np.all(np.abs(got - O_ref[others]) <= O_err[others]) and np.all(np.abs(got_lse - lse_ref[others]) <= lse_err[others])
    assert torch.allclose(O[others].float(), want[0][others].float(), atol=2e-2)
    b.table[1, 1] = b.k_pages.shape[0]                       # a page that is none, in the middle of what is seen
    b.masks[0][lone], b.tree[lone] = 0, 0
    b.v_pages[at(0, L - n + lone)[0], :, at(0, L - n + lone)[1]] = 0
    b.k_pages[at(0, L - n + lone)[0], :, at(0, L - n + lone)[1]] = 0
    check(b, max_new=max(news), name="page")


class TreeBatchWithout:
    """b without the keys of one token of sequence 0."""

    def __init__(self, b, token):
        self.__dict__.update(b.__dict__)
        self.b, self.at = b, b.lengths_list[0] - b.news[0] + token

    def sees(self, s, window=0):
        see = self.b.sees(s, window)
        if s == 0:
            see[:, self.at] = False
        return see

    def gathered(self, s):
        return self.b.gathered(s)


def test_values_beyond_the_sums_of_products():
    """Rows that see infinities have them (or NaN), the others of the item do not."""
    news = [60]
    b = TreeBatch([160], news, 4, 1, 64, seed=8, masks=[tree_mask(random_parents(random.Random(1), 60, roots=0.0))])
    seen_by = [t for t in range(60) if b.masks[0][t] >> 7 & 1]
    clean = run(b)
    page, row = int(b.table[0, (100 + 7) // 16]), (100 + 7) % 16
    b.v_pages[page, :, row] = float("inf")
    O, lse = run(b)
    rest = [t for t in range(60) if t not in seen_by]
    assert bool(torch.isinf(O[seen_by]).all()) and bool(torch.isfinite(O[rest]).all())
    assert torch.allclose(O[rest].float(), clean[0][rest].float(), atol=2e-2)


def test_layouts_outputs_and_rows_behind():
    b = TreeBatch([300, 77], [20, 33], 8, 2, 64, seed=3, packed=True, pool="seq", spare_rows=5, words=1)
    wide = torch.zeros(b.tree.shape[0], 3, dtype=torch.int64, device=DEV)
    wide[:, 1] = b.tree[:, 0]
    want = check(b)
    out, lse = torch.full(b.q.shape, 7.0, device=DEV), torch.full(b.q.shape[:2], 7.0, device=DEV)
    O, l = burst_paged_attention(b.q, *b.args(), scale=b.scale, tree=wide[:, 1:2], out=out, lse=lse)
    assert O is out and torch.equal(O[:53].to(BF16), want[0][:53]) and torch.equal(l[:53], want[1][:53])
    assert bool((out[53:] == 7).all()) and bool((lse[53:] == 7).all())
    full = check(b, full_p=True)
    assert torch.allclose(full[0][:53].float(), want[0][:53].float(), atol=2e-2)


def test_arrays_that_hold_anything_stay_inside():
    b = TreeBatch([300, 77, 9], [20, 33, 9], 8, 2, 64, seed=3)
    for lengths, starts, table in (([5, -3, 1 << 30], None, None), ([300, 77, 9], [0, 20, 53, 1 << 30], None), ([300, 77, 9], [-5, 20, 53, 62], None),
                                   ([300, 77, 9], [0, 40, 20, 62], None), ([300, 77, 9], None, 1 << 30)):
        t = b.table.clone() if table is None else torch.full_like(b.table, table)
        at = b.starts if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
        O, lse = burst_paged_attention(b.q, b.k_pages, b.v_pages, t, torch.tensor(lengths, dtype=torch.int32, device=DEV), at, tree=b.tree)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(O).all()) or starts is not None
    b.check(*run(b))


def test_repeated_and_captured_with_other_trees():
    b = TreeBatch([1500, 40, 700], [40, 40, 12], 8, 2, 128, seed=5)
    first = run(b)
    assert all(torch.equal(x, y) for x, y in zip(first, run(b)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = burst_paged_attention(b.q, *b.args(), scale=b.scale, tree=b.tree)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = burst_paged_attention(b.q, *b.args(), scale=b.scale, tree=b.tree)
    for seed in (6, 7, 8):
        c = TreeBatch([900 + seed, 40, 333], [40, 40, 12], 8, 2, 128, seed=seed)
        for name in ("q", "k_pages", "v_pages", "lengths", "starts", "tree"):
            if getattr(b, name).shape == getattr(c, name).shape:
                getattr(b, name).copy_(getattr(c, name))
        b.lengths_list, b.masks = c.lengths_list, c.masks
        graph.replay()
        want = run(b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), seed
        b.check(*out)


def test_errors():
    b = TreeBatch([30], [10], 4, 2, 64)
    for bad in (dict(tree=b.tree[:9]), dict(tree=b.tree.int()), dict(tree=b.tree.cpu()), dict(tree=b.tree[:, 0]), dict(tree=b.tree[:, :0]), dict(causal=False),
                dict(tree=b.tree.expand(10, 2)[:, :2])):
        with pytest.raises(ValueError):
            burst_paged_attention(b.q, *b.args(), **dict(dict(tree=b.tree), **bad))


def test_c_entry():
    """With a workspace of exactly the size that it asks for, between guards."""
    for dtype, H, news in ((BF16, 4, [1, 2]), (BF16, 4, [20, 31]), (BF16, 16, [20, 31]), (F32, 4, [20, 31]), (F32, 2, [1, 2])):
        b = TreeBatch([2000, 900], news, H, 2, 64, dtype=dtype, seed=1)
        T = sum(news)
        p = B.paged_params(T, H, 2, 64, dtype, b.k_pages, b.table, b.lengths, b.starts, scale=b.scale, max_new=max(news))
        O, lse = torch.full((T + 8, H, 64), 3.0, dtype=dtype, device=DEV), torch.full((T + 8, H), 3.0, device=DEV)
        need = B.burst_paged_workspace_bytes(p)
        ws = torch.full((need + 8192,), 77, dtype=torch.uint8, device=DEV)
        B.burst_paged_tree_fwd(b.q, b.k_pages, b.v_pages, O[4:-4], lse[4:-4], b.tree, p, ws[4096:4096 + need])
        b.check(O[4:-4], lse[4:-4])
        assert (ws[:4096] == 77).all() and (ws[4096 + need:] == 77).all()
        assert (O[:4] == 3).all() and (O[-4:] == 3).all() and (lse[:4] == 3).all() and (lse[-4:] == 3).all()
        with pytest.raises(B.BurstError):
            B.burst_paged_tree_fwd(b.q, b.k_pages, b.v_pages, O[4:-4], lse[4:-4], b.tree, p, ws[4096:4096 + need - 16])
