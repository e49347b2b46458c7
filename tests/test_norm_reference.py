"""The 64-bit gradients that the norm's tests compare with, against differences of the forward form."""
import numpy as np
import pytest

import norm_util as nu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(6, 6), (7, 4), (8, 0)])
def test_gradients_are_differences(d, dims, interleaved):
    rng = np.random.default_rng(d)
    x, g, w = rng.standard_normal((3, d)), rng.standard_normal((3, d)), 1 + rng.standard_normal(d) / 4
    pos = np.array([0, 17, 5000])
    how = dict(pos=pos, turns=np.array([0.11, 0.013, 0.0007])[:dims // 2], interleaved=interleaved, amplitude=1.3) if dims else {}
    eps, step = 1e-2, 1e-5
    dx, terms, _, _ = nu.backward(x, w, g, eps, **how)
    loss = lambda x, w: (nu.forward(x, w, eps, **how)[0] * g).sum()          # noqa: E731
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = step
        want = (loss(x + e, w) - loss(x - e, w)) / (2 * step)
        assert abs(dx[i] - want) < 1e-7 * (1 + abs(want)), i
    for c in range(d):
        e = np.zeros(d)
        e[c] = step
        want = (loss(x, w + e) - loss(x, w - e)) / (2 * step)
        assert abs(terms.sum(0)[c] - want) < 1e-7 * (1 + abs(want)), c
