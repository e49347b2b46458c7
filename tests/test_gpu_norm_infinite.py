"""Gradients that are not finite in columns that are not rotated: what they reach is what the formula says, and nothing else."""
import numpy as np
import pytest
import torch

import norm_util as nu
from paged_util import default_turns, f64
from paper_2403_09347_amd.rotary import burst_norm_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(128, 64), (128, 0), (64, 16), (96, 32), (7, 2), (3, 0)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_columns_that_are_not_rotated(dtype, interleaved, d, dims, value):
    gen = torch.Generator().manual_seed(d + dims)
    rand = lambda *s: torch.randn(s, generator=gen)           # noqa: E731
    x, g, w = rand(1, 3, 9, d).to(dtype).to(DEV).requires_grad_(True), rand(1, 3, 9, d).to(dtype).to(DEV), (1 + rand(d) / 8).to(DEV).requires_grad_(True)
    bad = [(0, 4, dims), (1, 2, d - 1), (2, 8, dims + (d - dims) // 2)]
    for h, row, c in bad:
        g[0, h, row, c] = value
    turns = default_turns(dims) if dims else None
    how = dict(pos=5 + np.arange(9)[None, None], turns=f64(turns), interleaved=interleaved) if dims else {}
    y = burst_norm_rotary(x, w, turns, 1e-6, 5, interleaved=interleaved)
    dx, dw = torch.autograd.grad(y, [x, w], g)
    with np.errstate(invalid="ignore", over="ignore"):
        want, terms, size, terms_size = nu.backward(f64(x), f64(w), f64(g), 1e-6, **how)
        got, want_w, got_w = f64(dx), terms.reshape(-1, d).sum(0), f64(dw)
    for a, b in ((got, want), (got_w, want_w)):
        assert np.array_equal(np.isnan(a), np.isnan(b))
        inf = np.isinf(b)
        assert np.array_equal(np.isinf(a), inf) and np.array_equal(a[inf], b[inf])
    rows = np.ones((3, 9), bool)
    for h, row, _ in bad:
        rows[h, row] = False
    assert np.isfinite(want[0][rows]).all() and not np.isfinite(want[0][~rows]).any()
    nu.near("dx", dx[0][torch.from_numpy(rows)], want[0][rows], size[0][rows])
    fine = np.isfinite(want_w)
    assert fine.sum() == d - len({c for _, _, c in bad})
    err = np.abs(got_w[fine] - want_w[fine])
    assert np.all(err <= (nu.unit(d) + 27 * 2.0 ** -24) * terms_size.reshape(-1, d).sum(0)[fine] + 2.0 ** -24 * 1.01 * np.abs(want_w[fine]))
