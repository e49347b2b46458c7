"""cos and sin of burst_rotary themselves: the rotation of (1, 0) and (0, 1) in fp32 gives them as they are.

The bound: half a step of fp32, 2^-24 of the value, and what 64 bits leave: the series' first missing terms (2^-37), and the fraction of a
turn, off by 2^-54 of a turn (and by 2^-44 in the 80 bits of the oracle, at positions below 2^20)."""
import numpy as np
import pytest
import torch

from paged_util import default_turns, f64
from paper_2403_09347_amd.paged import burst_cache_append
from paper_2403_09347_amd.rotary import burst_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def expected(pos, turns, amplitude, inverse=False):
    t = pos[:, None].astype(np.longdouble) * turns.astype(np.longdouble)
    ang = 2 * np.pi * (t - np.round(t)).astype(np.float64) * (-1 if inverse else 1)
    a = float(np.float32(amplitude))
    return a * np.cos(ang), a * np.sin(ang)


def check(got_c, got_s, pos, turns, amplitude, inverse=False):
    c, s = expected(pos, turns, amplitude, inverse)
    for name, got, want in (("cos", got_c, c), ("sin", got_s, s)):
        off = np.abs(got - want) - 2.0 ** -24 * np.abs(want)
        assert off.max() <= 2.0 ** -36 * amplitude, f"{name}: {np.abs(got - want).max():.3e} off"


@pytest.mark.parametrize("amplitude", [1.0, 1.2079441541679836])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("first", [0, 4096 * 7, (1 << 20) - 5000])
def test_rotation_and_gradient(first, interleaved, amplitude):
    N, d = 5000, 64
    x = torch.zeros(1, 2, N, d, device=DEV)                   # head 0: pairs (1, 0), head 1: (0, 1)
    a, b = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, d // 2), slice(d // 2, d))
    x[:, 0, :, a], x[:, 1, :, b] = 1, 1
    x.requires_grad_(True)
    turns = default_turns(d)
    y = burst_rotary(x, turns, first, interleaved=interleaved, amplitude=amplitude)
    (dx,) = torch.autograd.grad(y, x, x.detach())
    pos = first + np.arange(N)
    for out, inverse in ((f64(y), False), (f64(dx), True)):
        check(out[0, 0][:, a], out[0, 0][:, b], pos, f64(turns), amplitude, inverse)
        check(out[0, 1][:, b], -out[0, 1][:, a], pos, f64(turns), amplitude, inverse)


def test_quarters_and_their_halves():
    """Angles that are multiples of an eighth of a turn, and next to them."""
    steps = np.array([1 / 8 + k * e for k in range(-2, 3) for e in (2.0 ** -30, 2.0 ** -52, 1e-9)])
    turns = torch.tensor(steps, dtype=torch.float64, device=DEV)
    x = torch.zeros(1, 1, 64, 2 * len(steps), device=DEV)
    x[..., :len(steps)] = 1
    y = f64(burst_rotary(x, turns))[0, 0]
    check(y[:, :len(steps)], y[:, len(steps):], np.arange(64), steps, 1.0)


def test_appended_keys():
    n, d = 300, 32
    k = torch.zeros(n, 1, d, device=DEV)
    k[..., :d // 2] = 1
    pages = [torch.zeros(20, 1, 16, d, device=DEV) for _ in range(2)]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)   # noqa: E731
    turns = default_turns(d)
    burst_cache_append(k, k, *pages, torch.arange(20, dtype=torch.int32, device=DEV).view(1, 20), i32(n), i32(0, n), turns=turns,
                       offsets=torch.tensor([123457], device=DEV))
    got = f64(pages[0]).reshape(-1, d)[:n]
    check(got[:, :d // 2], got[:, d // 2:], 123457 + np.arange(n), f64(turns), 1.0)


def test_positions_far_beyond_any_context():
    """At 2^40 the fraction of a turn still has 2^-54: exact fractions by integers."""
    pos = (1 << 40) + np.arange(50)
    step = 3.0 ** -5
    frac = np.array([int(p) * int(step * 2 ** 60) % 2 ** 60 / 2 ** 60 for p in pos])               # (step is a multiple of 2^-60)
    x = torch.zeros(1, 1, 50, 2, device=DEV)
    x[..., 0] = 1
    y = f64(burst_rotary(x, torch.tensor([step], dtype=torch.float64, device=DEV), 1 << 40))[0, 0]
    for got, want in ((y[:, 0], np.cos(2 * np.pi * frac)), (y[:, 1], np.sin(2 * np.pi * frac))):
        assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -36)
