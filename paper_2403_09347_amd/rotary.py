"""Rotation of queries and keys by their positions, as models apply it before the attention: one differentiable torch call
for all tensors of a layer (native, csrc/burst_torch.cpp; the kernel is csrc/burst_rotary.hip), and the same with the norm that many
models put before it (csrc/burst_norm.hip)."""
import math

import torch

from . import binding as B


def rotary_turns(dims, base=10000.0, scaling=None, factor=1.0, original=4096, slow=1.0, fast=32.0, device="cuda"):
    """Turns per position of the dims / 2 pairs of columns, float64: base^(-2 i / dims) / 2 pi.  scaling, for contexts `factor` times
    longer than the model was trained for: "linear" (every pair `factor` times slower), "ntk" (a larger base, so that the slowest pair is
    `factor` times slower and the fastest as before) or "yarn" (pairs that turn less than `slow` times over the `original` length
    are `factor` times slower, those that turn more than `fast` times as before, in between in proportion; with
    rotary_amplitude(factor))."""
    if dims < 2 or dims % 2 or not base > 0 or not factor > 0:
        raise ValueError("dims: even, base and factor: positive expected")
    if scaling == "ntk" and dims > 2:
        base = base * factor ** (dims / (dims - 2))
    turns = base ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims) / (2 * math.pi)
    if scaling == "linear":
        turns = turns / factor
    elif scaling == "yarn":
        keep = ((original * turns - slow) / (fast - slow)).clamp(0, 1)
        turns = turns * keep + turns / factor * (1 - keep)
    elif scaling not in (None, "ntk"):
        raise ValueError("scaling: None, linear, ntk or yarn expected")
    return turns.to(device)


def rotary_amplitude(factor):
    """The factor of cos and sin that goes with "yarn"."""
    return 1.0 if factor <= 1 else 0.1 * math.log(factor) + 1.0


def burst_rotary(x, turns, offset=0, positions=None, interleaved=False, amplitude=1.0):
    """x: a [B, heads, rows, d] tensor or a list of them (bfloat16 or float32, d up to 128), rotated out of place by one launch (20 tensors each);
    returns a tensor or a list.  Row n is at position offset + n, or offset + positions[n] (positions: int64 [rows] or
    [B, rows]); offset and positions: one for all tensors, or a list.  turns: see rotary_turns; columns from 2 len(turns) on are copied.
    interleaved: columns 2 i and 2 i + 1 are a pair instead of i and i + len(turns).  Results lie in memory like x; views with
    a contiguous last dimension are read in place.  Gradients flow to x, rounded to its type; a captured backward pass to
    tensors that an earlier graph, made on the default stream, still holds is an error."""
    one = isinstance(x, torch.Tensor)
    xs = [x] if one else list(x)
    offsets = [int(o) for o in offset] if isinstance(offset, (list, tuple)) else [int(offset)] * len(xs)
    at = list(positions) if isinstance(positions, (list, tuple)) else [positions] * len(xs)
    try:
        y = B.load_torch_module().rotate(xs, turns, offsets, at, bool(interleaved), float(amplitude))
    except RuntimeError as e:
        raise B.from_native(e) from None
    return y[0] if one else y


def burst_norm_rotary(x, weights, turns=None, eps=1e-6, offset=0, positions=None, interleaved=False, amplitude=1.0):
    """x: a [B, heads, rows, d] tensor or a list of them (bfloat16 or float32, d from 2 to 128), every row divided by the root of its mean square
    (+ eps, positive: 2^-126 at least), multiplied by the weights [d] (of x's type or float32; one tensor for all, or a list with an entry for each, None: 1), and rotated as
    burst_rotary does (turns, offset, positions, interleaved, amplitude: see there; turns=None: not rotated), out of place, by one launch (12
    tensors each).  All of it in 32 bits (the angles in 64), rounded once; sums of squares beyond 32 bits' range count as infinite.  Returns a
    tensor or a list; results lie in memory like x.  Gradients flow to x and to the weights, whose gradients are summed in fp32 over all rows of all
    tensors that share them (the same tensor in the list) and rounded once; gradients of gradients are an error, and so is a captured backward pass
    to tensors that an earlier graph, made on the default stream, still holds."""
    one = isinstance(x, torch.Tensor)
    xs = [x] if one else list(x)
    ws = [weights] * len(xs) if weights is None or isinstance(weights, torch.Tensor) else list(weights)
    if len(ws) != len(xs):
        raise ValueError("one entry of weights per tensor expected")
    each, weight_of = [], []
    for w in ws:
        at = -1 if w is None else next((i for i, e in enumerate(each) if e is w), len(each))
        if at == len(each):
            each.append(w)
        weight_of.append(at)
    offsets = [int(o) for o in offset] if isinstance(offset, (list, tuple)) else [int(offset)] * len(xs)
    at = list(positions) if isinstance(positions, (list, tuple)) else [positions] * len(xs)
    try:
        y = B.load_torch_module().norm_rotate(xs, each, weight_of, turns, float(eps), offsets, at, bool(interleaved), float(amplitude))
    except RuntimeError as e:
        raise B.from_native(e) from None
    return y[0] if one else y
