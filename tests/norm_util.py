"""The plain 64-bit forms of rows normalised, weighted and rotated, and of their gradients, with the bounds of 32-bit errors."""
import numpy as np

from paged_util import HALF, f64, rotation


def forward(x, w, eps, pos=None, turns=None, interleaved=False, amplitude=1.0):
    """x [..., d], w [d] (or 1), positions [...] as numpy: (y, sizes: what rounding of a value is relative to)."""
    x = np.asarray(x, np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    if turns is None:
        return n, np.abs(n)
    y, size = rotation(n, pos, turns, interleaved, amplitude)
    size[..., :2 * len(turns)] *= abs(amplitude)
    return y, size


def backward(x, w, g, eps, pos=None, turns=None, interleaved=False, amplitude=1.0):
    """(dx, terms of dw [..., d], sizes of both)."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    h, h_size = g.copy(), np.abs(g)
    if turns is not None:
        h, h_size = rotation(g, pos, turns, interleaved, amplitude, inverse=True)
        h_size[..., :2 * len(turns)] *= abs(amplitude)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, u_size = h * w, h_size * np.abs(w)
    dx = r * (u - x * r * r * (u * x).mean(-1, keepdims=True))
    dx_size = r * (u_size + np.abs(x) * r * r * (u_size * np.abs(x)).mean(-1, keepdims=True))
    return dx, h * x * r, dx_size, h_size * np.abs(x) * r


def unit(d):
    """Relative error of 32-bit results beside their own rounding: sums of d squares (and of d products) one after the other, a root, a reciprocal, cos and sin, half a
    dozen products."""
    return (2 * d + 32) * 2.0 ** -24


def near(name, got, want, size, more=0.0):
    """Rounded once to its type; `more`: error beside that, relative to `size`."""
    got_ = f64(got)
    err = np.abs(got_ - want)
    bound = HALF[got.dtype] * np.abs(want) * 1.01 + (unit(want.shape[-1]) + more) * size + 1e-30
    assert np.all(np.isfinite(got_)), f"{name}: not finite"
    assert np.all(err <= bound), f"{name}: {np.max(err - bound):.3e} over its bound, error {err.max():.3e}"


def check_forward(name, y, x, w, eps, pos=None, turns=None, interleaved=False, amplitude=1.0):
    want, size = forward(f64(x), 1.0 if w is None else f64(w), eps, pos, turns, interleaved, amplitude)
    near(name, y, want, size)


def check_dx(name, dx, x, w, g, eps, pos=None, turns=None, interleaved=False, amplitude=1.0):
    want, _, size, _ = backward(f64(x), 1.0 if w is None else f64(w), f64(g), eps, pos, turns, interleaved, amplitude)
    near(name, dx, want, size)


def dw_terms(x, w, g, eps, pos=None, turns=None, interleaved=False, amplitude=1.0):
    """(sum of the terms of dw, of their sizes, number of rows), to be added up over the tensors that share a weight."""
    _, terms, _, size = backward(f64(x), f64(w), f64(g), eps, pos, turns, interleaved, amplitude)
    d = terms.shape[-1]
    return terms.reshape(-1, d).sum(0), size.reshape(-1, d).sum(0), terms.size // d


def check_dw(name, dw, parts):
    want, size, rows = (sum(p[i] for p in parts) for i in range(3))
    near(name, dw, want, size, rows * 2.0 ** -24)              # (a sum of `rows` terms in 32 bits, in any order)
