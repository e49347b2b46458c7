"""burst_rotary: the rotation and its gradient against 64 bits, layouts, odd sizes, positions far out; burst_attention with it."""
import numpy as np
import pytest
import torch

from oracle import burst_oracle as orc
from paged_util import check_rotation, default_turns, f64
from paper_2403_09347_amd import workloads
from paper_2403_09347_amd.autograd import burst_attention
from paper_2403_09347_amd.rotary import burst_rotary, rotary_amplitude, rotary_turns

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def rand(*shape, dtype=F32, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(128, 128), (128, 64), (64, 64), (96, 96), (96, 48), (80, 40), (80, 32), (32, 16), (24, 2), (7, 6), (2, 2), (126, 126)])
def test_values_and_gradients(dtype, interleaved, d, dims):
    B, H, N, off = 2, 3, 37, 5000
    x = rand(B, H, N, d, dtype=dtype, seed=d + dims).requires_grad_(True)
    g = rand(B, H, N, d, dtype=dtype, seed=1)
    turns = default_turns(dims)
    y = burst_rotary(x, turns, off, interleaved=interleaved, amplitude=1.25)
    (dx,) = torch.autograd.grad(y, x, g)
    pos = off + np.arange(N)[None, None]
    check_rotation("y", y, x, pos, f64(turns), interleaved, 1.25)
    check_rotation("dx", dx, g, pos, f64(turns), interleaved, 1.25, inverse=True)


@pytest.mark.parametrize("N", [0, 1, 2, 15, 16, 17, 100, 1000])
@pytest.mark.parametrize("H", [1, 8, 33])
def test_lengths(N, H):
    x = rand(1, H, N, 128, dtype=BF16)
    y = burst_rotary(x, default_turns(128), 7)
    assert y.shape == x.shape
    if N:
        check_rotation("y", y, x, 7 + np.arange(N)[None, None], f64(default_turns(128)))


@pytest.mark.parametrize("layout", ["seq", "packed", "expanded", "odd"])
def test_layouts_are_read_in_place_and_kept(layout):
    base = rand(2, 4, 50, 64, dtype=BF16)
    if layout == "expanded":
        x = base[:, :1].expand(2, 4, 50, 64)
    elif layout == "odd":                                     # rows that start anywhere
        x = rand(2, 4, 50, 67, dtype=BF16)[..., 1:65]
    else:
        x = workloads.relayout(base, layout)
    y = burst_rotary(x, default_turns(64), 3)
    check_rotation("y", y, x, 3 + np.arange(50)[None, None], f64(default_turns(64)))
    if layout == "seq":
        assert y.stride() == x.stride()


def test_far_positions_of_any_order():
    x = rand(2, 3, 64, 64, seed=3)
    pos = torch.randint(0, 1 << 24, (2, 64), generator=torch.Generator().manual_seed(1)).to(DEV)
    pos[0, 0], pos[0, 1], pos[1, 5] = -5, 0, (1 << 31) + 12345
    turns = default_turns(64)
    y = burst_rotary(x, turns, 100, positions=pos)
    check_rotation("y", y, x, 100 + f64(pos)[:, None], f64(turns))
    one = burst_rotary(x, turns, positions=pos[0])             # [rows], for every batch entry
    check_rotation("one", one, x, f64(pos[0])[None, None], f64(turns))
    every = burst_rotary(x, turns, positions=pos[:, ::2].repeat_interleave(2, 1))
    check_rotation("copied", every, x, f64(pos[:, ::2].repeat_interleave(2, 1))[:, None], f64(turns))


def test_several_tensors_and_more_than_one_launch_takes():
    xs = [rand(1, 1 + i % 3, 5 + i, 32, dtype=BF16, seed=i).requires_grad_(i % 4 != 1) for i in range(45)]
    xs[7] = xs[7][:, :, :0]
    turns = default_turns(32)
    ys = burst_rotary(xs, turns, offset=[10 * i for i in range(45)])
    for i, (x, y) in enumerate(zip(xs, ys)):
        if x.numel():
            check_rotation(f"y{i}", y, x, 10 * i + np.arange(x.shape[2])[None, None], f64(turns))
    leaves = [x for x in xs if x.requires_grad and x.is_leaf]
    used = [y for x, y in zip(xs, ys) if x.requires_grad and x.is_leaf][::2]
    gs = [torch.randn_like(y) for y in used]
    grads = torch.autograd.grad(used, leaves[::2], gs)
    for x, g, dx in zip(leaves[::2], gs, grads):
        i = next(i for i, t in enumerate(xs) if t is x)
        check_rotation(f"dx{i}", dx, g, 10 * i + np.arange(x.shape[2])[None, None], f64(turns), inverse=True)


def test_gradient_against_differences():
    """The rotation is linear: a difference quotient has rounding errors only.  Sums of 2 x 3 x 9 x 32 products of values of size 1 and
    differences of outputs of size 10: 1728 x 10 x 2^-22 bounds both."""
    x, u, g = rand(2, 3, 9, 32, seed=1), rand(2, 3, 9, 32, seed=2), rand(2, 3, 9, 32, seed=3)
    f = lambda t: f64(burst_rotary(t, default_turns(32), 12345))
    leaf = x.clone().requires_grad_(True)
    y = burst_rotary(leaf, default_turns(32), 12345)
    (dx,) = torch.autograd.grad(y, leaf, g)
    quotient = (f(x + u) - f(x - u)) / 2
    assert abs((quotient * f64(g)).sum() - (f64(dx) * f64(u)).sum()) <= 1728 * 10 * 2.0 ** -22


def test_gradients_of_gradients():
    """The gradient is linear in what it is given: its gradient turns forward again."""
    x, g, u = (rand(1, 2, 11, 32, seed=i).requires_grad_(i < 2) for i in range(3))
    pos = torch.randint(0, 1 << 20, (11,), generator=torch.Generator().manual_seed(3)).to(DEV)
    y = burst_rotary([x, x.detach()], default_turns(32), 5, positions=[pos, None], interleaved=True)
    (dx,) = torch.autograd.grad(y[0], x, g, create_graph=True)
    check_rotation("dx", dx, g, 5 + f64(pos)[None, None], f64(default_turns(32)), True, inverse=True)
    (dg,) = torch.autograd.grad(dx, g, u)
    check_rotation("dg", dg, u, 5 + f64(pos)[None, None], f64(default_turns(32)), True)


def test_the_graph_is_freed_kept_and_guarded_as_torchs_own():
    x, t = rand(1, 2, 9, 16).requires_grad_(True), default_turns(16)
    pos = torch.arange(9, device=DEV)
    y = burst_rotary(x, t, positions=pos)
    one, two = (torch.autograd.grad(y, x, torch.ones_like(y), retain_graph=True)[0] for _ in range(2))
    assert torch.equal(one, two)
    torch.autograd.grad(y, x, torch.ones_like(y))
    with pytest.raises(RuntimeError):                         # freed
        torch.autograd.grad(y, x, torch.ones_like(y))
    y = burst_rotary(x, t, positions=pos)
    pos.add_(1)
    with pytest.raises(RuntimeError):                         # changed in place
        torch.autograd.grad(y, x, torch.ones_like(y))
    with torch.no_grad():
        assert not burst_rotary(x, t).requires_grad
    assert not burst_rotary(x.detach(), t).requires_grad
    a, b = burst_rotary([x, x.detach()], t)
    a.sum().backward()                                        # one of two outputs used
    assert x.grad is not None


def test_captured_gradients():
    """Forward and backward recorded together, replayed with other inputs and eager work in between."""
    x, g, t = rand(1, 4, 200, 64, dtype=BF16).requires_grad_(True), rand(1, 4, 200, 64, dtype=BF16, seed=2), default_turns(64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(burst_rotary(x, t, 9), x, g)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = burst_rotary(x, t, 9)
        (dx,) = torch.autograd.grad(y, x, g)
    for seed in (3, 4, 5):
        with torch.no_grad():
            x.copy_(rand(1, 4, 200, 64, dtype=BF16, seed=seed))
        g.copy_(rand(1, 4, 200, 64, dtype=BF16, seed=seed + 10))
        graph.replay()
        torch.cuda.synchronize()
        check_rotation("y", y, x, 9 + np.arange(200)[None, None], f64(t))
        check_rotation("dx", dx, g, 9 + np.arange(200)[None, None], f64(t), inverse=True)


def test_a_gradient_of_a_sum():
    """Its gradient is one value seen everywhere, with strides of 0."""
    x = rand(1, 2, 9, 16).requires_grad_(True)
    burst_rotary(x, default_turns(16)).sum().backward()
    check_rotation("dx", x.grad, torch.ones_like(x), np.arange(9)[None, None], f64(default_turns(16)), inverse=True)


def test_refusals():
    x, t = rand(1, 2, 3, 64), default_turns(64)
    for bad in (dict(x=x.half()), dict(x=x[0]), dict(x=[x, x.to(BF16)]), dict(x=[x, x[..., :32]]), dict(turns=t.float()), dict(turns=t.cpu()),
                dict(turns=default_turns(66)), dict(turns=t[:0]), dict(turns=t[::2]), dict(turns=t.clone().requires_grad_(True)),
                dict(positions=torch.arange(4, device=DEV)), dict(positions=torch.arange(3)), dict(positions=torch.arange(3, device=DEV).int()),
                dict(positions=torch.zeros(2, 3, dtype=torch.int64, device=DEV)), dict(offset=[1, 2]), dict(amplitude=float("nan"))):
        with pytest.raises((ValueError, RuntimeError)):
            burst_rotary(**dict(dict(x=x, turns=t), **bad))


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0)])
def test_scaled_frequencies(scaling, factor):
    t0, t = rotary_turns(64, device="cpu"), rotary_turns(64, scaling=scaling, factor=factor, device="cpu")
    if scaling == "linear":
        assert torch.allclose(t * factor, t0, rtol=1e-15)
    elif scaling == "ntk":
        assert torch.allclose(t[0], t0[0], rtol=1e-15) and torch.allclose(t[-1] * factor, t0[-1], rtol=1e-12)
    else:
        assert torch.equal(t[4096 * t0 > 32], t0[4096 * t0 > 32]) and torch.allclose(t[4096 * t0 < 1] * factor, t0[4096 * t0 < 1], rtol=1e-15)
        assert abs(rotary_amplitude(factor) - (0.1 * np.log(16) + 1)) < 1e-12
    x = rand(1, 2, 20, 64)
    check_rotation("y", burst_rotary(x, t.to(DEV), 9), x, 9 + np.arange(20)[None, None], f64(t))


def test_other_stream_and_captured_replays():
    x, turns = rand(1, 4, 300, 128, dtype=BF16), default_turns(128)
    want = burst_rotary(x, turns, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = burst_rotary(x, turns, 5)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    pos = torch.arange(300, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = burst_rotary(x, turns, positions=pos)
    for k in (1, 40, 7):
        pos.copy_(torch.arange(300, device=DEV) * k)
        x.copy_(rand(1, 4, 300, 128, dtype=BF16, seed=k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, burst_rotary(x, turns, positions=pos))


@pytest.mark.parametrize("dtype,H,KV,d,tol", [(F32, 2, 2, 40, 1e-4), (BF16, 4, 2, 64, 2e-2)])
def test_attention_of_rotated_rows(dtype, H, KV, d, tol):
    """burst_attention(turns=...) against the oracle on rows rotated in 64 bits, with the gradients brought back.  Tolerances: the
    benchmark statement's, as in the other parity tests, and for bf16 twice that for the additional rounding of q, k and
    of their gradients."""
    Nq, rows, off = 70, [64, 50], 44
    name = "bf16" if dtype == BF16 else "f32"
    case = workloads.make_case(1, H, d, Nq, rows, name, seed=5, device=DEV, causal=True, q_off=off, kv_heads=KV)
    turns = default_turns(d)
    leaves = [t.requires_grad_(True) for t in [case["Q"], *case["K"], *case["V"]]]
    O, lse = burst_attention(case["Q"], case["K"], case["V"], case["scale"], True, off, turns=turns)
    grads = torch.autograd.grad(O, leaves, case["dO"])
    from paged_util import rotation
    qp, kp, tn = off + np.arange(Nq), np.arange(sum(rows)), f64(turns)
    dK, dV = np.zeros((KV, sum(rows), d)), np.zeros((KV, sum(rows), d))
    limit = tol * (2 if dtype == BF16 else 1)
    for h in range(H):
        q, _ = rotation(f64(case["Q"][0, h]), qp, tn)
        k0 = np.concatenate([f64(t[0, h * KV // H]) for t in case["K"]])
        v = np.concatenate([f64(t[0, h * KV // H]) for t in case["V"]])
        k, _ = rotation(k0, kp, tn)
        dO = f64(case["dO"][0, h])
        O_ref, lse_ref = orc.full_forward(q, k, v, case["scale"], True, qp, kp)
        assert np.abs(f64(O[0, h]) - O_ref).max() <= limit and np.abs(f64(lse[0, h]) - lse_ref).max() <= limit
        dq, dk, dv = orc.full_backward(q, k, v, dO, case["scale"], True, qp, kp)
        assert np.abs(f64(grads[0][0, h]) - rotation(dq, qp, tn, inverse=True)[0]).max() <= limit * max(1, np.abs(dq).max())
        dK[h * KV // H] += rotation(dk, kp, tn, inverse=True)[0]
        dV[h * KV // H] += dv
    gK = np.concatenate([f64(t[0]) for t in grads[1:3]], 1)
    gV = np.concatenate([f64(t[0]) for t in grads[3:5]], 1)
    assert np.abs(gK - dK).max() <= limit * max(1, np.abs(dK).max()) and np.abs(gV - dV).max() <= limit * max(1, np.abs(dV).max())


def test_a_rotated_ring_is_the_rotated_sequence():
    """The last device's rows of a ring, chunk by chunk, and the whole sequence in one chunk see the same positions."""
    q, k, v = (rand(1, 2, 256, 64, dtype=BF16, seed=i) for i in range(3))
    turns = default_turns(64)
    whole, _ = burst_attention(q, [k], [v], causal=True, turns=turns)
    last, _ = burst_attention(q[:, :, 192:], list(k.split(64, 2)), list(v.split(64, 2)), causal=True, q_off=192, turns=turns)
    assert (whole[:, :, 192:].float() - last.float()).abs().max().item() <= 2e-2


def test_more_rows_than_a_launch_has_blocks_for():
    rows, t = (1 << 27) + 100, default_turns(2)
    x = (torch.arange(2 * rows, device=DEV) % 251).to(BF16).view(1, 1, rows, 2)
    y = burst_rotary(x, t)
    for at in (0, (1 << 27) - 50, rows - 50):
        check_rotation(at, y[:, :, at:at + 50], x[:, :, at:at + 50], at + np.arange(50)[None, None], f64(t))
