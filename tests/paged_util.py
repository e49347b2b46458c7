"""Batches of sequences with paged caches, and the plain 64-bit forms of the rotation, of appending and of attention over pages."""
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative to the value


def rotation(x, pos, turns, interleaved=False, amplitude=1.0, inverse=False):
    """x [..., d] and positions [...] as numpy; (result, |a| + |b| of the pairs) in 64 bits."""
    x, pos, turns = np.asarray(x, np.float64), np.asarray(pos, np.float64), np.asarray(turns, np.float64)
    n = len(turns)
    i, j = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    # (80 bits: a product in 64 is off by up to 2^-53 of itself, 10^-6 of an angle at position 2^33, which the kernel's fma is not)
    t = pos[..., None].astype(np.longdouble) * turns.astype(np.longdouble)
    ang = 2 * np.pi * (t - np.round(t)).astype(np.float64) * (-1 if inverse else 1)
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
    y, size = x.copy(), np.abs(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return y, size


def check_rotation(name, got, x, pos, turns, interleaved=False, amplitude=1.0, inverse=False):
    """Rounding to the type, cos and sin to 2^-22 (32-bit series and angle), and two products and a sum in 32 bits; the columns past the
    pairs bit for bit."""
    want, size = rotation(f64(x), pos, turns, interleaved, amplitude, inverse)
    err = np.abs(f64(got) - want)
    bound = HALF[got.dtype] * np.abs(want) * (1 + 2.0 ** -7) + 2.0 ** -21 * abs(amplitude) * size
    assert np.all(err <= bound), f"{name}: {np.max(err - bound):.3e} over the bound"
    n = 2 * len(turns)
    assert torch.equal(got[..., n:], x[..., n:]), name


def f64(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """lengths[s] tokens of sequence s, the last news[s] of them new; their pages in random places of the pools."""

    def __init__(self, lengths, news, H, KV, d, page=16, dtype=torch.bfloat16, seed=0, pool="head", packed=False, spare_rows=0, spare_pages=2,
                 scale_qk=1.0, device="cuda"):
        self.lengths_list, self.news, self.H, self.KV, self.d, self.page, self.dtype = list(lengths), list(news), H, KV, d, page, dtype
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen).to(dtype).to(device)   # noqa: E731
        S, T = len(lengths), sum(news) + spare_rows
        if packed:
            qkv = rand(T, H + 2 * KV, d)
            qkv[:, :H] *= scale_qk
            self.q, self.k, self.v = qkv.split([H, KV, KV], dim=1)
        else:
            self.q, self.k, self.v = rand(T, H, d) * scale_qk, rand(T, KV, d), rand(T, KV, d)
        per = [-(-n // page) for n in lengths]
        pages = sum(per) + spare_pages
        mk = (lambda: rand(pages, page, KV, d).transpose(1, 2)) if pool == "seq" else (lambda: rand(pages, KV, page, d))
        self.k_pages, self.v_pages = mk(), mk()
        order = torch.randperm(pages, generator=gen).to(torch.int32)
        self.table = torch.full((S, max(per + [1])), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(per):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.free = order[at:].tolist()
        self.table = self.table.to(device)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=device)
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device=device)
        self.scale = d ** -0.5

    def args(self):
        return self.k_pages, self.v_pages, self.table, self.lengths, self.starts

    def positions(self):
        """(sequence, position) of every new token."""
        return [(s, self.lengths_list[s] - n + t) for s, n in enumerate(self.news) for t in range(n)]

    def gathered(self, s):
        """Keys and values of a sequence, [KV, len, d] in 64 bits, and which of its pages are pages."""
        n, page = self.lengths_list[s], self.page
        ids = self.table[s].cpu().numpy()[:-(-n // page)]
        ok = (ids >= 0) & (ids < self.k_pages.shape[0])
        idx = torch.from_numpy(np.where(ok, ids, 0)).long().to(self.k_pages.device)
        take = lambda p: f64(p[idx]).transpose(1, 0, 2, 3).reshape(self.KV, -1, self.d)[:, :n]   # noqa: E731
        return take(self.k_pages), take(self.v_pages), np.repeat(ok, page)[:n]

    def reference(self, causal=True, window=0):
        """O, lse and the bounds of their errors, per new token and head."""
        T = sum(self.news)
        O, lse = np.zeros((T, self.H, self.d)), np.full((T, self.H), -np.inf)
        O_err, lse_err = np.zeros_like(O), np.zeros_like(lse)
        q = f64(self.q)
        group, at = self.H // self.KV, 0
        half = HALF[self.dtype]
        for s, n in enumerate(self.news):
            L = self.lengths_list[s]
            K, V, ok = self.gathered(s)
            pos, key = np.arange(L - n, L)[:, None], np.arange(L)[None]
            see = np.broadcast_to(ok[None], (n, L)).copy()
            if causal:
                see &= key <= pos
            if window:
                see &= key > pos - window
            for h in range(self.H if L else 0):
                k, v, x = K[h // group], V[h // group], q[at:at + n, h]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = np.where(see, (x @ k.T) * self.scale, -np.inf)
                    most = np.where(see, (np.abs(x) @ np.abs(k).T) * self.scale, 0).max(-1, initial=0)
                    m = z.max(-1, initial=-np.inf)
                    p = np.exp(z - np.where(np.isfinite(m), m, 0)[:, None])
                    l = p.sum(-1)
                    some = l > 0
                    vis = np.where(see[..., None], v[None], 0) if not np.isfinite(v).all() else None
                    pv = p @ v if vis is None else np.einsum("ij,ijk->ik", np.where(see, p, 0), vis)
                    pa = p @ np.abs(v) if vis is None else np.einsum("ij,ijk->ik", np.where(see, p, 0), np.abs(vis))
                    inv = np.where(some, 1 / np.where(some, l, 1), 0)[:, None]
                O[at:at + n, h] = np.where(some[:, None], pv * inv, 0)
                lse[at:at + n, h] = np.where(some, m + np.log(np.where(some, l, 1)), -np.inf)
                # scores: d products and the scale in 32 bits; exponents of up to 2 `most`; l and O: sums of L terms in 32 bits
                e = (self.d + 16) * 2.0 ** -24 * most + 2.0 ** -20
                long = L * 2.0 ** -24
                rounded = 2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0     # of P
                O_err[at:at + n, h] = (rounded + 4 * e + 2 * long)[:, None] * pa * inv + half * np.abs(O[at:at + n, h]) * 1.01 + 1e-30
                lse_err[at:at + n, h] = np.where(some, 2 * e + long + 2.0 ** -22 * (np.abs(np.where(some, lse[at:at + n, h], 0)) + most), 0)
            at += n
        return O, lse, O_err, lse_err

    def check(self, O, lse, causal=True, window=0, name=""):
        T = sum(self.news)
        O_ref, lse_ref, O_err, lse_err = self.reference(causal, window)
        got, got_lse = f64(O[:T]), f64(lse[:T])
        none = np.isneginf(lse_ref)
        assert np.array_equal(np.isneginf(got_lse), none), name + ": rows that see nothing"
        assert np.all(np.isfinite(got)) and np.all(np.isfinite(got_lse[~none])), name + ": not finite"
        err = np.abs(got - O_ref)
        assert np.all(err <= O_err), f"{name}: O {np.max(err - O_err):.3e} over its bound, error {err.max():.3e}"
        err = np.abs(np.where(none, 0, got_lse - np.where(none, 0, lse_ref)))
        assert np.all(err <= lse_err), f"{name}: lse {np.max(err - lse_err):.3e} over its bound, error {err.max():.3e}"


def default_turns(dims, device="cuda"):
    return (10000.0 ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims) / (2 * math.pi)).to(device)
