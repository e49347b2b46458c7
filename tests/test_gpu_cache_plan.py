"""burst_cache_plan against the same books kept on the host: enough of everything, too few pages or rows, ended sequences, arrays that hold anything."""
import random

import numpy as np
import pytest
import torch

import plan_util
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_plan

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def case(S, page, width, pages, most_new, seed, ended=0.1, trees=False, filled=0.5, words=1, junk=False, wide=0):
    rng = random.Random(seed)
    cap = width * page
    lengths = [rng.randrange(int(cap * filled) + 1) for _ in range(S)]
    new = [-1 if rng.random() < ended else rng.choice([0, 1, rng.randrange(most_new + 1)]) for _ in range(S)]
    order = list(range(pages))
    rng.shuffle(order)
    table = np.full((S, width), -1, np.int64)
    for s in range(S):
        for c in range(-(-lengths[s] // page)):
            table[s, c] = order.pop() if order else -1
    free = order + [rng.randrange(pages) for _ in range(pages - len(order))]
    count = len(order)
    parents = None
    if trees:
        parents = np.array([[rng.randrange(-1, t + 1) if rng.random() < 0.95 else rng.choice([t, t + 5, -7, 1 << 30]) for t in range(most_new + wide)] for _ in range(S)])
    if junk:
        lengths = [rng.choice([n, -5, cap, cap - 1, cap + 3, 2 ** 31 - 1, 1 << 30]) for n in lengths]
        new = [rng.choice([n, 2 ** 31 - 1, -2 ** 31, 1 << 20, cap]) if rng.random() < 0.3 else n for n in new]
        for _ in range(S * width // 5):
            table[rng.randrange(S), rng.randrange(width)] = rng.choice([-9, pages, 2 ** 31 - 1, -2 ** 31])
        for _ in range(pages // 4):
            free[rng.randrange(pages)] = rng.choice([-1, pages, 2 ** 31 - 1])
        count = rng.choice([count, count + pages, -3, 0])
    return dict(new=new, lengths=lengths, table=table, free=free, count=count, page=page, parents=parents, words=words)


def check(c, rows, strided=False):
    want = plan_util.plan(rows=rows, **c)
    table, free, count = i32(c["table"]), i32(c["free"]), i32([c["count"]])
    if strided:
        wide = torch.full((table.shape[0], table.shape[1] + 7), 77, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        table = wide[:, :table.shape[1]]
    parents = None if c["parents"] is None else i32(c["parents"])
    for again in range(2):                                    # the same call again changes nothing
        got = burst_cache_plan(i32(c["new"]), i32(c["lengths"]), table, free, count, c["page"], rows, parents, c["words"])
        torch.cuda.synchronize()
        enough = all(n <= 0 or b - a == n for n, a, b in zip(c["new"], want[0], want[0][1:]))
        if again and not enough:
            break
        for name, g, w in zip(("starts", "lengths", "slots", "positions", "tree"), got, want):
            assert (g is None) == (w is None), name
            if g is not None:
                assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape)), (name, again)
        assert np.array_equal(table.cpu().numpy(), want[5]), ("table", again)
        assert free.tolist() == want[6] and count.tolist() == [want[7]], ("stack", again)
    if strided:
        assert bool((wide[:, table.shape[1]:] == 77).all())
    return want


@pytest.mark.parametrize("S,page,width,most", [(1, 16, 1, 1), (3, 16, 5, 40), (64, 16, 40, 9), (65, 32, 9, 64), (500, 64, 8, 3), (1025, 16, 3, 5), (4096, 16, 2, 2)])
@pytest.mark.parametrize("trees", [False, True])
def test_enough_of_everything(S, page, width, most, trees):
    for seed in range(3):
        c = case(S, page, width, S * width + 1, most, seed, trees=trees)
        rows = sum(max(n, 0) for n in c["new"]) + seed * 3
        want = check(c, rows, strided=seed == 1)
        if seed == 0 and all(max(n, 0) + l <= width * page for n, l in zip(c["new"], c["lengths"])):
            assert want[0][-1] == rows


def test_no_sequences_and_no_rows():
    got = burst_cache_plan(i32([]), i32([]), torch.zeros(0, 4, dtype=torch.int32, device=DEV), i32([1, 2]), i32([2]), 16, 5)
    assert got.starts.tolist() == [0] and got.slots.tolist() == got.positions.tolist() == [-1] * 5 and got.tree is None
    check(case(7, 16, 4, 40, 3, 1), 0)


def test_long_prompts_and_many_rows():
    """Prompts through thousands of pages beside single tokens: more entries than the threads have at a time, and rows of a second launch."""
    for seed, (S, page, most, rows) in enumerate([(5, 16, 60000, 150000), (300, 16, 900, 90000), (40, 128, 3000, 40000), (4096, 16, 60, 100000)]):
        c = case(S, page, -(-2 * most // page), S * (-(-2 * most // page)), most, seed, filled=0.4, trees=False)
        check(c, rows)


def test_too_few_pages_or_rows():
    for seed in range(12):
        rng = random.Random(seed)
        S = rng.choice([4, 70, 300])
        c = case(S, 16, 12, rng.choice([3, 2 * S, 7 * S]), 60, seed, trees=seed % 2 == 0)
        for rows in (rng.randrange(200), 100 * S):
            check(c, rows)


@pytest.mark.parametrize("words,most", [(1, 64), (2, 128), (3, 200), (4, 256), (2, 300)])
def test_masks(words, most):
    """Trees of as many tokens as there are bits and more (chunks); parents that are none of the tokens before; columns of parents fewer and more than tokens."""
    for wide in (-3, 0, 5):
        for seed in range(2):
            c = case(40, 16, 60, 40 * 60, most, seed, trees=True, words=words, wide=wide)
            check(c, sum(max(n, 0) for n in c["new"]) + 2)
    chain = dict(case(3, 16, 60, 180, 4, 0, ended=0), new=[64 * words, 1, 64 * words - 1], lengths=[0, 5, 17], words=words)
    chain["parents"] = np.array([[t - 1 for t in range(64 * words)]] * 3)
    want = check(chain, 128 * words)
    assert want[3][:64 * words] == list(range(64 * words))


def test_arrays_that_hold_anything():
    for seed in range(30):
        rng = random.Random(100 + seed)
        c = case(rng.choice([1, 5, 200]), rng.choice([16, 64]), rng.randrange(1, 20), rng.randrange(1, 900), 50, seed, trees=seed % 3 == 0, words=rng.choice([1, 2]), junk=True)
        check(c, rng.choice([0, 1, 100, 4000]))


def test_pages_that_come_back_are_given_again():
    """A stack without pages: what the ended sequences have is enough."""
    table = np.array([[3, 1, -1], [0, -1, -1], [-1, -1, -1], [2, -1, -1]])
    c = dict(new=[-1, 1, 20, -1], lengths=[30, 16, 0, 9], table=table, free=[9, 9, 9, 9], count=0, page=16, parents=None, words=1)
    want = check(c, 21)
    assert want[5].tolist() == [[-1, -1, -1], [0, 2, -1], [1, 3, -1], [-1, -1, -1]] and want[7] == 0 and want[0] == [0, 0, 1, 21, 21]


def test_captured_with_other_contents():
    cs = [case(90, 16, 30, 90 * 30, 64, seed, trees=True) for seed in range(4)]
    rows = 3000
    names = ("new", "lengths", "table", "free", "parents")
    t = {n: i32(cs[0][n]) for n in names}
    count = i32([cs[0]["count"]])
    call = lambda: burst_cache_plan(t["new"], t["lengths"], t["table"], t["free"], count, 16, rows, t["parents"])   # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for c in cs[1:]:
        for n in names:
            t[n].copy_(i32(c[n]))
        count.copy_(i32([c["count"]]))
        graph.replay()
        torch.cuda.synchronize()
        want = plan_util.plan(rows=rows, **c)
        for g, w in zip(out, want):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape))
        assert np.array_equal(t["table"].cpu().numpy(), want[5]) and count.tolist() == [want[7]]


def test_errors():
    new, lengths, table, free, count = i32([1, 2]), i32([0, 0]), i32([[-1], [-1]]), i32([0, 1, 2]), i32([3])
    good = dict(new=new, lengths=lengths, table=table, free=free, count=count, page=16, rows=3)
    burst_cache_plan(**good)
    for bad in (dict(new=new.long()), dict(new=new[:1]), dict(lengths=lengths.cpu()), dict(table=table[0]), dict(table=table[:1]), dict(free=table), dict(count=new), dict(rows=-1),
                dict(rows=1 << 20), dict(page=8), dict(page=24), dict(page=1 << 30), dict(free=free[::2]), dict(table=table.expand(2, 5)), dict(parents=table.long()), dict(parents=table[:1]),
                dict(parents=table.clone(), words=0), dict(parents=table), dict(parents=free[:2, None]), dict(free=lengths), dict(table=table[:, :0], page=0)):
        with pytest.raises((ValueError, B.BurstError)):
            burst_cache_plan(**dict(good, **bad))
    version = table._version
    burst_cache_plan(**good)
    assert table._version > version


def test_c_entry():
    c = case(9, 16, 6, 60, 30, 4, trees=True)
    rows = 200
    want = plan_util.plan(rows=rows, **c)
    table, free, count = i32(c["table"]), i32(c["free"]), i32([c["count"]])
    out = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (10, 9)] + [torch.empty(rows, dtype=torch.int64, device=DEV) for _ in range(2)]
    tree = torch.empty(rows, 1, dtype=torch.int64, device=DEV)
    B.burst_cache_plan(i32(c["new"]), i32(c["lengths"]), table, free, count, 16, *out, i32(c["parents"]), tree)
    for g, w in zip(out + [tree, table], list(want[:4]) + [want[4], want[5]]):
        assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape))
