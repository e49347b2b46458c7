"""Serving with drafted tokens, all calls together: plan, append (norms, rotation, slots, positions), attention with masks, keep; what stays in the cache
and what every step answers are those of plain attention over the tokens that were kept."""
import random

import numpy as np
import pytest
import torch

import norm_util as nu
import plan_util
from paged_util import HALF, f64
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_cache_keep, burst_cache_plan
from paper_2403_09347_amd.rotary import rotary_turns
from tree_util import branch, random_parents

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, KV, D, PAGE, EPS = 4, 2, 64, 16, 1e-5


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("captured", [False, True])
def test_steps(dtype, captured):
    rng, gen = random.Random(5), torch.Generator().manual_seed(5)
    S, width, pages, rows, most, layers = 4, 12, 30, 160, 64, 2
    rand = lambda *s: torch.randn(s, generator=gen).to(dtype).to(DEV)          # noqa: E731
    weights = [(1 + torch.randn(D, generator=gen) / 4).to(DEV) for _ in range(2)]
    turns = rotary_turns(D, base=500.0, device=DEV)
    pools = [(torch.zeros(pages, KV, PAGE, D, dtype=dtype, device=DEV), torch.zeros(pages, KV, PAGE, D, dtype=dtype, device=DEV)) for _ in range(layers)]
    walks = [PagedWalk(k, v, D ** -0.5, turns, norms=weights, eps=EPS) for k, v in pools]
    table, free, count = torch.full((S, width), -1, dtype=torch.int32, device=DEV), i32(range(pages)), i32([pages])
    lengths, new, parents = i32([0] * S), i32([0] * S), i32(np.full((S, most), -1))
    kept, counts = i32(np.zeros((S, most))), i32([0] * S)
    tokens = [[rand(rows, h, D) for h in (H, KV, KV)] for _ in range(layers)]
    history = [[[] for _ in range(S)] for _ in range(layers)]                  # (k, v) of every token that stays, 64 bits

    def step():
        plan = burst_cache_plan(new, lengths, table, free, count, PAGE, rows, parents)
        return plan, [w.planned_step(*t, table, plan) for w, t in zip(walks, tokens)]

    def settle(plan):
        lengths.copy_(burst_cache_keep([k for k, _ in pools], [v for _, v in pools], table, plan.lengths, plan.starts, kept, counts))

    graph = out = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            settle(step()[0])
        torch.cuda.current_stream().wait_stream(side)
        graph, last = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        with torch.cuda.graph(last):
            settle(out[0])
    # prompts (one of more tokens than a mask has bits), then trees, a sequence that ends, another in its place
    for news in ([70, 9, 1, 33], [12, 40, 3, 1], [20, 1, 0, 7], [5, -1, 30, 9], [1, 25, 8, 12]):
        ups = [random_parents(rng, n, roots=0) if 0 < n <= 12 else [t - 1 for t in range(n)] for n in news]
        picks = [list(range(n)) if n > 12 else branch(u, rng.randrange(n)) if n > 0 else [] for n, u in zip(news, ups)]
        new.copy_(i32(news))
        parents.copy_(i32([u[:most] + [-1] * (most - len(u[:most])) for u in ups]))
        kept.copy_(i32([(p + [0] * most)[:most] for p in picks]))
        counts.copy_(i32([len(p) for p in picks]))
        if max(len(p) for p in picks) > most:                                  # (a prompt is kept whole: its places are right as they are)
            counts.copy_(i32([min(len(p), most) for p in picks]))
        for t in tokens:
            for x in t:
                x.copy_(rand(*x.shape))
        want_plan = plan_util.plan(news, lengths.tolist(), table.cpu().numpy(), free.tolist(), int(count[0]), PAGE, rows, [u + [-1] * most for u in ups])
        if captured:
            graph.replay()
            plan, results = out
        else:
            plan, results = step()
        torch.cuda.synchronize()
        for g, w in zip(plan, want_plan):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape))
        for layer in range(layers):
            q, k, v = (f64(x) for x in tokens[layer])
            pos = np.array(want_plan[3])[:, None]
            how = dict(pos=pos, turns=f64(turns))
            qn = nu.forward(q, f64(weights[0]), EPS, **how)[0]
            kn = nu.forward(k, f64(weights[1]), EPS, **how)[0]
            O, lse = (f64(x) for x in results[layer])
            row = 0
            for s, n in enumerate(news):
                if n < 0:
                    history[layer][s] = []
                for t in range(max(n, 0)):
                    path = branch(ups[s], t)
                    K = np.array([x[0] for x in history[layer][s]] + [kn[row + j] for j in path])
                    V = np.array([x[1] for x in history[layer][s]] + [v[row + j] for j in path])
                    assert pos[row + t, 0] == len(K) - 1
                    for h in range(H):
                        z = K[:, h // (H // KV)] @ qn[row + t, h] * D ** -0.5
                        p = np.exp(z - z.max())
                        ref = p @ V[:, h // (H // KV)] / p.sum()
                        # Half steps of q, k (twice in a score), P and O; an error e of all scores is one of 2 e in O, e in lse.
                        half, size = HALF[dtype], (np.abs(K[:, h // (H // KV)]) @ np.abs(qn[row + t, h])).max() * D ** -0.5
                        e = 2 * half * size + 2 * nu.unit(D) * size + 2.0 ** -18
                        assert np.abs(O[row + t, h] - ref).max() <= (2 * e + 2 * half) * 1.02 * np.abs(V).max(), (news, s, t, h)
                        assert abs(lse[row + t, h] - (z.max() + np.log(p.sum()))) <= e * 1.02
                history[layer][s] += [(kn[row + j], v[row + j]) for j in picks[s]]
                row += max(n, 0)
        if captured:
            last.replay()
        else:
            settle(plan)
        torch.cuda.synchronize()
        if max(len(p) for p in picks) > most:
            lengths.copy_(i32([len(h) for h in history[0]]))
        assert lengths.tolist() == [len(h) for h in history[0]]
        held = table.cpu().numpy()
        for layer in range(layers):
            for s in range(S):
                for p, (k, v) in enumerate(history[layer][s]):
                    got_k, got_v = (f64(pool[int(held[s, p // PAGE]), :, p % PAGE]) for pool in pools[layer])
                    assert np.abs(got_k - k).max() <= (HALF[dtype] * 1.02 + 2 * nu.unit(D)) * np.abs(k).max() and np.abs(got_v - v).max() == 0
