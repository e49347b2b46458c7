"""Batches with trees of drafted tokens: their masks, and the plain 64-bit form of attention over them."""
import random

import numpy as np
import torch

from paged_util import HALF, Batch, f64


def branch(parents, t):
    path = []
    while t >= 0:
        path.append(t)
        t = parents[t]
    return path[::-1]


def random_parents(rng, n, bushy=4, roots=0.05):
    return [-1 if t == 0 or rng.random() < roots else rng.randrange(max(0, t - bushy), t) for t in range(n)]


def tree_mask(parents):
    return [sum(1 << j for j in branch(parents, t)) for t in range(len(parents))]


def as_words(masks, words):
    """Python integers as an int64 array [rows, words]."""
    out = np.zeros((len(masks), words), np.uint64)
    for i, m in enumerate(masks):
        for w in range(words):
            out[i, w] = (m >> (64 * w)) & ((1 << 64) - 1)
    return out.view(np.int64)


class TreeBatch(Batch):
    """masks[s]: for every new token of a sequence the integer whose bits are the new tokens that it sees; None: random trees."""

    def __init__(self, lengths, news, *args, words=1, masks=None, junk=False, device="cuda", **kw):
        super().__init__(lengths, news, *args, device=device, **kw)
        rng = random.Random(kw.get("seed", 0) + 17)
        self.words = words
        self.masks = masks or [tree_mask(random_parents(rng, n)) if n <= 64 * words else [0] * n for n in news]
        spare = self.q.shape[0] - sum(news)
        junk_bits = lambda n: rng.getrandbits(64 * words) >> n << n if junk and n < 64 * words else 0   # noqa: E731
        rows = [m | junk_bits(n) for n, ms in zip(news, self.masks) for m in ms] + [rng.getrandbits(64 * words) for _ in range(spare)]
        self.tree = torch.from_numpy(as_words(rows, words)).to(device) if rows else torch.zeros(0, words, dtype=torch.int64, device=device)

    def sees(self, s, window=0):
        """[new tokens, keys] of a sequence, pages aside."""
        n, L = self.news[s], self.lengths_list[s]
        key = np.arange(L)[None]
        if n > 64 * self.words:
            pos = np.arange(L - n, L)[:, None]
            return (key <= pos) & ((key > pos - window) if window else True)
        see = np.zeros((n, L), bool)
        for t, m in enumerate(self.masks[s]):
            m &= (1 << n) - 1
            base = L - n
            first = max(0, base + bin(m).count("1") - 1 - window + 1) if window else 0
            see[t, first:max(base, 0)] = True
            for j in range(n):
                if m >> j & 1 and base + j >= 0:
                    see[t, base + j] = True
        return see

    def reference(self, causal=True, window=0):
        T = sum(self.news)
        O, lse = np.zeros((T, self.H, self.d)), np.full((T, self.H), -np.inf)
        O_err, lse_err = np.zeros_like(O), np.zeros_like(lse)
        q, group, at, half = f64(self.q), self.H // self.KV, 0, HALF[self.dtype]
        for s, n in enumerate(self.news):
            L = self.lengths_list[s]
            K, V, ok = self.gathered(s)
            see = self.sees(s, window) & ok[None]
            for h in range(self.H if L else 0):
                k, v, x = np.where(see.any(0)[:, None], K[h // group], 0), np.where(see.any(0)[:, None], V[h // group], 0), q[at:at + n, h]
                z = np.where(see, (x @ k.T) * self.scale, -np.inf)
                most = np.where(see, (np.abs(x) @ np.abs(k).T) * self.scale, 0).max(-1, initial=0)
                m = z.max(-1, initial=-np.inf)
                p = np.exp(z - np.where(np.isfinite(m), m, 0)[:, None])
                l = p.sum(-1)
                some = l > 0
                inv = np.where(some, 1 / np.where(some, l, 1), 0)[:, None]
                O[at:at + n, h] = p @ v * inv
                lse[at:at + n, h] = np.where(some, m + np.log(np.where(some, l, 1)), -np.inf)
                # (see Batch.reference: scores, exponents, sums in 32 bits, P rounded, O rounded once)
                e = (self.d + 16) * 2.0 ** -24 * most + 2.0 ** -20
                long = L * 2.0 ** -24
                rounded = 2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0
                O_err[at:at + n, h] = (rounded + 4 * e + 2 * long)[:, None] * (p @ np.abs(v)) * inv + half * np.abs(O[at:at + n, h]) * 1.01 + 1e-30
                lse_err[at:at + n, h] = np.where(some, 2 * e + long + 2.0 ** -22 * (np.abs(np.where(some, lse[at:at + n, h], 0)) + most), 0)
            at += n
        return O, lse, O_err, lse_err
