"""Plans for attention with a window: masks of the last tokens of every branch, and steps of drafted tokens that see what the same tokens see as a prompt's chunk or one by one."""
import random

import numpy as np
import pytest
import torch

import plan_util
from paged_util import HALF, f64
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_cache_plan
from tree_util import as_words, branch, random_parents

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 16


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def columns(ups, most):
    return i32([u[:most] + [-1] * (most - len(u[:most])) for u in ups])


@pytest.mark.parametrize("words,many", [(1, False), (1, True), (2, False), (3, False), (3, True)])
@pytest.mark.parametrize("window", [1, 2, 5, 31, 32, 63, 64, 65, 100, 1 << 31])
def test_masks(words, many, window):
    rng, S = random.Random(window + words), 60 if many else 12
    news = [rng.choice([1, 2, 40, 63, 64, 65, 64 * words, rng.randrange(1, 64 * words + 1)]) for _ in range(S)]
    ups = [random_parents(rng, n, bushy=rng.choice([1, 1, 2, 8]), roots=rng.choice([0, 0.05])) for n in news]
    rows, pages, width, most = sum(news) + 3, 60 * S, 60, max(news)
    table = np.full((S, width), -1)
    want = plan_util.plan(news, [7 * s for s in range(S)], table, list(range(pages)), pages, PAGE, rows, [u + [-1] * (most - len(u)) for u in ups], words)
    masks = [sum(1 << j for j in branch(u, t)[-window:]) if n <= 64 * words else 0 for n, u in zip(news, ups) for t in range(n)] + [0] * 3
    for entry in ("torch", "C"):
        if entry == "C" and window > 0x7fffffff:
            continue
        args = (i32(news), i32([7 * s for s in range(S)]), i32(table), i32(range(pages)), i32([pages]), PAGE)
        if entry == "torch":
            got = burst_cache_plan(*args, rows, columns(ups, most), words, window)
        else:
            got = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (S + 1, S)] + [torch.empty(rows, dtype=torch.int64, device=DEV) for _ in range(2)]
            got.append(torch.empty(rows, words, dtype=torch.int64, device=DEV))
            B.burst_cache_plan(*args, *got[:4], columns(ups, most), got[4], window)
        for g, w in zip(got, want[:4]):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w)), entry
        assert np.array_equal(got[4].cpu().numpy(), as_words(masks, words)), entry


def plain(q, keys, values, scale):
    """(O, lse, bounds of both) of one query head over what it sees, in 64 bits (errors as Batch.reference has them)."""
    z, d = keys @ q * scale, len(q)
    p = np.exp(z - z.max())
    O, most = p @ values / p.sum(), (np.abs(keys) @ np.abs(q)).max() * scale
    e, long = (d + 16) * 2.0 ** -24 * most + 2.0 ** -20, len(z) * 2.0 ** -24
    lse = z.max() + np.log(p.sum())
    return O, lse, (4 * e + 2 * long) * (p @ np.abs(values)) / p.sum(), p @ np.abs(values) / p.sum(), 2 * e + long + 2.0 ** -22 * (abs(lse) + most)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window", [1, 3, 16, 40, 70, 90, 500])
@pytest.mark.parametrize("shape", ["chains", "trees"])
def test_steps(dtype, window, shape):
    """Drafted tokens behind contexts of 0 to 150 tokens; chains also as chunks (no parents) and token by token, whose answers are held to the same values."""
    H, KV, d, words = 4, 2, 64, 2
    rng, gen = random.Random(window), torch.Generator().manual_seed(window)
    rand = lambda *s: torch.randn(s, generator=gen).to(dtype).to(DEV)          # noqa: E731
    contexts, news = [0, 5, 33, 150], [128, 60, 90, 17]
    S, T, width = 4, sum(news), 20
    ups = [list(range(-1, n - 1)) if shape == "chains" else random_parents(rng, n, bushy=2, roots=0.03) for n in news]
    before, now = [rand(sum(contexts), h, d) for h in (H, KV, KV)], [rand(T, h, d) for h in (H, KV, KV)]
    walk, table, free, count = None, None, None, None

    def fresh():
        nonlocal walk, table, free, count
        walk = PagedWalk(*(torch.zeros(S * width, KV, PAGE, d, dtype=dtype, device=DEV) for _ in range(2)), d ** -0.5, window=window)
        table, free, count = torch.full((S, width), -1, dtype=torch.int32, device=DEV), i32(range(S * width)), i32([S * width])
        walk.planned_step(*before, table, burst_cache_plan(i32(contexts), i32([0] * S), table, free, count, PAGE, sum(contexts)))

    answers = {}
    fresh()
    plan = burst_cache_plan(i32(news), i32(contexts), table, free, count, PAGE, T, columns(ups, max(news)), words, window)
    answers["tree"] = walk.planned_step(*now, table, plan)
    if shape == "chains":
        fresh()
        answers["chunk"] = walk.planned_step(*now, table, burst_cache_plan(i32(news), i32(contexts), table, free, count, PAGE, T))
        fresh()
        firsts = np.concatenate([[0], np.cumsum(news)])
        O, lse = torch.empty(T, H, d, dtype=dtype, device=DEV), torch.empty(T, H, device=DEV)
        for t in range(max(news)):
            rows = [int(firsts[s] + t) for s in range(S) if t < news[s]]
            one = burst_cache_plan(i32([int(t < n) for n in news]), i32([c + min(t, n) for c, n in zip(contexts, news)]), table, free, count, PAGE, len(rows))
            O[rows], lse[rows] = walk.planned_step(*(x[rows] for x in now), table, one)
        answers["one by one"] = O, lse
    (_, bk, bv), (q, k, v) = ([f64(x) for x in l] for l in (before, now))
    row = old = 0
    half = HALF[dtype]
    results = {name: (f64(O), f64(lse)) for name, (O, lse) in answers.items()}
    for s, n in enumerate(news):
        for t in range(n):
            path = [row + j for j in branch(ups[s], t)]
            K = np.concatenate([bk[old:old + contexts[s]], k[path]])[-window:]
            V = np.concatenate([bv[old:old + contexts[s]], v[path]])[-window:]
            for h in range(H):
                ref, l, e, size, l_err = plain(q[row + t, h], K[:, h // 2], V[:, h // 2], d ** -0.5)
                bound = e + (2.0 ** -8 if dtype == torch.bfloat16 else 0) * size + half * 1.01 * np.abs(ref) + 1e-30
                for name, (O, lse) in results.items():
                    assert np.all(np.abs(O[row + t, h] - ref) <= bound), (name, s, t, h)
                    assert abs(lse[row + t, h] - l) <= l_err, (name, s, t, h)
        row += n
        old += contexts[s]
