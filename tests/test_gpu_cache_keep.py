"""burst_cache_keep against moves on the host."""
import random

import pytest
import torch

from paged_util import Batch
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_keep

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make(lengths, news, layers=1, KV=2, d=64, seed=0, **kw):
    bs = [Batch(lengths, news, KV, KV, d, seed=seed, **kw)]
    for i in range(1, layers):
        b = Batch(lengths, news, KV, KV, d, seed=seed + i, **kw)
        bs.append(b)
    return bs


def kept_lists(news, seed, share=0.4):
    rng = random.Random(seed)
    return [sorted(rng.sample(range(n), rng.choice([0, n, int(n * share), min(n, 1)]))) for n in news]


def tensors(kept, most=None, fill=-9):
    most = max([len(k) for k in kept] + [1]) if most is None else most
    return i32([k + [fill] * (most - len(k)) for k in kept]), i32([len(k) for k in kept])


def moved(b, pool, kept):
    """The pool with the kept rows moved, in increasing order."""
    out, table = pool.clone(), b.table.cpu().numpy()
    for s, (n, L) in enumerate(zip(b.news, b.lengths_list)):
        at = lambda p: (int(table[s, p // b.page]), p % b.page)   # noqa: E731
        for j, k in enumerate(kept[s]):
            if L - n + j < 0:
                continue
            (fp, fr), (tp, tr) = at(L - n + k), at(L - n + j)
            if fp >= 0 and tp >= 0 and fp < pool.shape[0] and tp < pool.shape[0]:
                out[tp, :, tr] = pool[fp, :, fr]
    return out


def check(bs, kept, most=None):
    b = bs[0]
    before = [(x.k_pages.clone(), x.v_pages.clone()) for x in bs]
    k, counts = tensors(kept, most)
    got = burst_cache_keep([x.k_pages for x in bs], [x.v_pages for x in bs], b.table, b.lengths, b.starts, k, counts)
    torch.cuda.synchronize()
    assert got.tolist() == [L - n + len(x) for L, n, x in zip(b.lengths_list, b.news, kept)] and got.dtype == torch.int32
    for x, (kb, vb) in zip(bs, before):
        assert torch.equal(x.k_pages, moved(b, kb, kept)) and torch.equal(x.v_pages, moved(b, vb, kept))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 8), (F32, 64), (F32, 4), (BF16, 96)])
@pytest.mark.parametrize("pool", ["head", "seq"])
def test_moves(dtype, d, pool):
    for seed, (lengths, news) in enumerate([([40, 5, 64, 7, 100], [12, 5, 64, 1, 0]), ([300, 77], [70, 33]), ([1], [1])]):
        bs = make(lengths, news, 3, d=d, dtype=dtype, pool=pool, seed=10 * seed)
        check(bs, kept_lists(news, seed))


def test_more_tokens_than_a_list_and_more_tensors_than_a_launch():
    news = [900, 257, 256]
    check(make([1000, 257, 300], news, KV=1, d=8), kept_lists(news, 1, 0.9))
    check(make([1000, 257, 300], news, KV=1, d=8), [list(range(1, 900)), list(range(257)), [255]])
    bs = make([20, 9], [8, 9], 203, KV=1, d=8)
    check(bs, [[0, 3, 7], [1, 2, 8]], most=5)


def test_rows_that_start_anywhere():
    """Pools whose rows are not on 16 bytes: element by element."""
    for dtype, d in ((BF16, 8), (F32, 4)):
        b = make([40, 30], [20, 30], d=d, dtype=dtype)[0]
        for name in ("k_pages", "v_pages"):
            wide = torch.zeros(*getattr(b, name).shape[:3], d + 3, dtype=dtype, device=DEV)
            wide[..., 1:d + 1] = getattr(b, name)
            setattr(b, name, wide[..., 1:d + 1])
        check([b], [[0, 2, 9, 19], [5, 6, 7, 29]])


def test_places_without_a_page():
    b = make([40, 40], [30, 30])[0]
    b.table[0, 1], b.table[1, 2] = -1, b.k_pages.shape[0]
    check([b], [[0, 3, 9, 25, 28], [1, 2, 22, 23, 29]])


def test_anything_in_the_lists_stays_among_the_new_tokens():
    news, lengths = [20, 7, 3], [50, 7, 100]
    for seed in range(8):
        rng = random.Random(seed)
        b = make(lengths, news, seed=seed)[0]
        kept = [[rng.choice([rng.randrange(n), -1, n, n + 5, 2 ** 31 - 1, -2 ** 31]) for _ in range(n)] for n in news]
        counts = [rng.choice([n, -4, 2 ** 31 - 1, 0]) for n in news]
        before = [b.k_pages.clone(), b.v_pages.clone()]
        k, _ = tensors(kept)
        got = burst_cache_keep(b.k_pages, b.v_pages, b.table, b.lengths, b.starts, k, i32(counts))
        assert got.tolist() == [L - n + min(max(c, 0), n) for L, n, c in zip(lengths, news, counts)]
        table = b.table.cpu().numpy()
        for pool, old in zip((b.k_pages, b.v_pages), before):
            same = (pool == old)
            for s, (n, L) in enumerate(zip(news, lengths)):
                rows = [(int(table[s, p // 16]), p % 16) for p in range(L - n, L)]
                held = torch.stack([old[p, :, r] for p, r in rows])
                for p, r in rows:
                    assert any(torch.equal(pool[p, :, r], h) for h in held)
                    same[p, :, r] = True
            assert bool(same.all())
    for lengths_, starts in (([5, -9, 1 << 30], [0, 20, 27, 30]), ([50, 7, 100], [7, 3, 1 << 30, -5])):
        burst_cache_keep(b.k_pages, b.v_pages, b.table, i32(lengths_), i32(starts), k, i32(counts))
        torch.cuda.synchronize()


def test_nothing_is_kept():
    b = make([40, 9], [20, 9])[0]
    before = [b.k_pages.clone(), b.v_pages.clone()]
    for kept, counts in ((torch.zeros(2, 0, dtype=torch.int32, device=DEV), i32([5, 0])), (i32([[3], [1]]), i32([0, 0]))):
        assert burst_cache_keep(b.k_pages, b.v_pages, b.table, b.lengths, b.starts, kept, counts).tolist() == [20, 0]
        assert torch.equal(b.k_pages, before[0]) and torch.equal(b.v_pages, before[1])
    none = torch.zeros(0, 2, 16, 64, dtype=BF16, device=DEV)
    assert burst_cache_keep(none, none, b.table, b.lengths, b.starts, i32([[3], [1]]), i32([1, 1])).tolist() == [21, 1]


def test_captured():
    news, lengths = [20, 33], [60, 33]
    b = make(lengths, news)[0]
    k, counts = i32([[0] * 33] * 2), i32([0, 0])
    call = lambda: burst_cache_keep(b.k_pages, b.v_pages, b.table, b.lengths, b.starts, k, counts)   # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (1, 2, 3):
        kept = kept_lists(news, seed)
        x, c = tensors(kept, 33)
        k.copy_(x)
        counts.copy_(c)
        want = moved(b, b.k_pages, kept), moved(b, b.v_pages, kept)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.k_pages, want[0]) and torch.equal(b.v_pages, want[1]) and out.tolist() == [L - n + len(x) for L, n, x in zip(lengths, news, kept)]


def test_errors():
    a, b = make([30], [10]), make([30], [10], d=32)
    x = a[0]
    k, counts = i32([[0, 2]]), i32([2])
    good = dict(k_pages=x.k_pages, v_pages=x.v_pages, table=x.table, lengths=x.lengths, starts=x.starts, kept=k, counts=counts)
    for bad in (dict(k_pages=[x.k_pages, b[0].k_pages], v_pages=[x.v_pages, b[0].v_pages]), dict(k_pages=[], v_pages=[]), dict(k_pages=[x.k_pages] * 2), dict(v_pages=x.k_pages),
                dict(k_pages=[x.k_pages] * 2, v_pages=[x.v_pages] * 2), dict(kept=k.long()), dict(kept=k[0]), dict(counts=counts.cpu()), dict(counts=i32([1, 2])),
                dict(k_pages=x.k_pages.clone().requires_grad_(True)), dict(kept=k.expand(3, 2)), dict(starts=x.starts[:1])):
        with pytest.raises((ValueError, B.BurstError)):
            burst_cache_keep(**dict(good, **bad))
    version = x.v_pages._version
    burst_cache_keep(**good)
    assert x.v_pages._version > version


def test_c_entry():
    b = make([40, 9], [20, 9])[0]
    kept = [[1, 5, 6], [0, 8]]
    k, counts = tensors(kept)
    want = moved(b, b.k_pages, kept), moved(b, b.v_pages, kept)
    p = B.paged_params(29, 2, 2, 64, BF16, b.k_pages, b.table, b.lengths, b.starts)
    out = torch.empty_like(b.lengths)
    B.burst_cache_keep([b.k_pages, b.v_pages], k, counts, out, p)
    assert torch.equal(b.k_pages, want[0]) and torch.equal(b.v_pages, want[1]) and out.tolist() == [23, 2]
