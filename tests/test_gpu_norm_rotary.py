"""burst_norm_rotary: values and gradients against 64 bits, layouts, odd sizes, shared weights, rows with zeros and infinities; burst_attention with it."""
import numpy as np
import pytest
import torch

import norm_util as nu
from paged_util import default_turns, f64
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd import workloads
from paper_2403_09347_amd.autograd import burst_attention
from paper_2403_09347_amd.rotary import burst_norm_rotary, burst_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def rand(*shape, dtype=F32, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def weight(d, dtype=F32, seed=0):
    return (1 + rand(d, seed=seed + 100) / 4).to(dtype)


def check_all(x, w, g, y, grads, pos=None, turns=None, eps=EPS, interleaved=False, amplitude=1.0):
    how = dict(pos=pos, turns=None if turns is None else f64(turns), interleaved=interleaved, amplitude=amplitude)
    nu.check_forward("y", y, x, w, eps, **how)
    nu.check_dx("dx", grads[0], x, w, g, eps, **how)
    if w is not None:
        assert grads[1].dtype == w.dtype and grads[1].shape == w.shape
        nu.check_dw("dw", grads[1], [nu.dw_terms(x, w, g, eps, **how)])


@pytest.mark.parametrize("dtype,wtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(128, 128), (128, 64), (128, 8), (64, 64), (96, 96), (96, 48), (80, 40), (80, 32), (32, 16), (24, 2), (7, 6), (2, 2), (126, 126), (120, 2)])
def test_values_and_gradients(dtype, wtype, interleaved, d, dims):
    N, off = 37, 5000
    x = rand(2, 3, N, d, dtype=dtype, seed=d + dims).requires_grad_(True)
    g, w = rand(2, 3, N, d, dtype=dtype, seed=1), weight(d, wtype).requires_grad_(True)
    turns = default_turns(dims)
    y = burst_norm_rotary(x, w, turns, EPS, off, interleaved=interleaved, amplitude=1.25)
    check_all(x, w, g, y, torch.autograd.grad(y, [x, w], g), off + np.arange(N)[None, None], turns, EPS, interleaved, 1.25)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [2, 3, 40, 64, 100, 128])
def test_without_rotation_and_without_weights(dtype, d):
    x, g, w = rand(1, 5, 33, d, dtype=dtype).requires_grad_(True), rand(1, 5, 33, d, dtype=dtype, seed=1), weight(d).requires_grad_(True)
    y = burst_norm_rotary(x, w, eps=1e-2)
    check_all(x, w, g, y, torch.autograd.grad(y, [x, w], g), eps=1e-2)
    y = burst_norm_rotary(x, None, eps=1e-2)
    check_all(x, None, g, y, torch.autograd.grad(y, [x], g), eps=1e-2)


@pytest.mark.parametrize("N", [0, 1, 2, 15, 16, 17, 100, 1000])
@pytest.mark.parametrize("H", [1, 8, 33])
def test_lengths(N, H):
    x, g, w = rand(1, H, N, 128, dtype=BF16).requires_grad_(True), rand(1, H, N, 128, dtype=BF16, seed=1), weight(128, BF16).requires_grad_(True)
    turns = default_turns(128)
    y = burst_norm_rotary(x, w, turns, EPS, 7)
    dx, dw = torch.autograd.grad(y, [x, w], g)
    assert y.shape == dx.shape == x.shape
    if N:
        check_all(x, w, g, y, (dx, dw), 7 + np.arange(N)[None, None], turns)
    else:
        assert torch.equal(dw, torch.zeros_like(dw))


@pytest.mark.parametrize("N", [9000, 40000])
def test_many_rows_a_workgroup(N):
    """More tiles than the gradient has workgroups: each goes through several."""
    x, g, w = rand(2, 9, N, 32, dtype=BF16).requires_grad_(True), rand(2, 9, N, 32, dtype=BF16, seed=1), weight(32).requires_grad_(True)
    turns = default_turns(32)
    y = burst_norm_rotary(x, w, turns, EPS)
    check_all(x, w, g, y, torch.autograd.grad(y, [x, w], g), np.arange(N)[None, None], turns)


@pytest.mark.parametrize("layout", ["seq", "packed", "expanded", "odd", "heads"])
def test_layouts_are_read_in_place_and_kept(layout):
    base = rand(2, 4, 50, 64, dtype=BF16)
    if layout == "expanded":
        x = base[:, :1].expand(2, 4, 50, 64)
    elif layout == "odd":                                     # rows that start anywhere
        x = rand(2, 4, 50, 67, dtype=BF16)[..., 1:65]
    elif layout == "heads":                                   # 8-byte granules alone
        x = rand(2, 4, 50, 68, dtype=BF16)[..., 4:]
    else:
        x = workloads.relayout(base, layout)
    x = x.detach().requires_grad_(True)
    w, turns, g = weight(64, BF16).requires_grad_(True), default_turns(64), rand(2, 50, 4, 64, dtype=BF16, seed=3).transpose(1, 2)
    y = burst_norm_rotary(x, w, turns, EPS, 3)
    check_all(x, w, g, y, torch.autograd.grad(y, [x, w], g), 3 + np.arange(50)[None, None], turns)
    if layout == "seq":
        assert y.stride() == x.stride()
    y = burst_norm_rotary(x, w, turns, EPS, 3)
    (dx,) = torch.autograd.grad(y.sum(), x)                   # (a gradient that is one value for all)
    nu.check_dx("dx", dx, x, w, torch.ones_like(g), EPS, pos=3 + np.arange(50)[None, None], turns=f64(turns))


def test_gradients_of_broadcast_heads_and_of_strided_weights():
    one = rand(2, 1, 40, 64).requires_grad_(True)
    both = weight(128).requires_grad_(True)
    x, w, turns, g = one.expand(2, 6, 40, 64), both[::2], default_turns(64), rand(2, 6, 40, 64, seed=2)
    y = burst_norm_rotary(x, w, turns)
    dx, dw = torch.autograd.grad(y, [one, both], g)
    want, _, size, _ = nu.backward(f64(x), f64(w), f64(g), EPS, np.arange(40)[None, None], f64(turns))
    nu.near("dx", dx, want.sum(1, keepdims=True), size.sum(1, keepdims=True), 6 * 2.0 ** -23)
    nu.check_dw("dw", dw[::2], [nu.dw_terms(x, w, g, EPS, np.arange(40)[None, None], f64(turns))])
    assert torch.equal(dw[1::2], torch.zeros_like(dw[1::2]))


def test_far_positions_of_any_order():
    x, w, turns = rand(2, 3, 64, 64, seed=3), weight(64), default_turns(64)
    pos = torch.randint(0, 1 << 24, (2, 64), generator=torch.Generator().manual_seed(1)).to(DEV)
    pos[0, 0], pos[0, 1], pos[1, 5] = -5, 0, (1 << 31) + 12345
    nu.check_forward("y", burst_norm_rotary(x, w, turns, EPS, 100, positions=pos), x, w, EPS, 100 + f64(pos)[:, None], f64(turns))
    nu.check_forward("one", burst_norm_rotary(x, w, turns, EPS, positions=pos[0]), x, w, EPS, f64(pos[0])[None, None], f64(turns))


def test_several_tensors_with_shared_weights_and_more_than_one_launch_takes():
    n, turns = 30, default_turns(32)
    xs = [rand(1, 1 + i % 3, 5 + i, 32, dtype=BF16, seed=i).requires_grad_(i % 4 != 1) for i in range(n)]
    xs[7] = xs[7][:, :, :0]
    gs = [rand(*x.shape, dtype=BF16, seed=50 + i) for i, x in enumerate(xs)]
    each = [weight(32, BF16, 0).requires_grad_(True), weight(32, F32, 1).requires_grad_(True), weight(32, BF16, 2)]
    of = [(0, 1, 0, 2, None)[i % 5] for i in range(n)]
    ws = [None if k is None else each[k] for k in of]
    ys = burst_norm_rotary(xs, ws, turns, EPS, offset=[10 * i for i in range(n)])
    at = [10 * i + np.arange(x.shape[2])[None, None] for i, x in enumerate(xs)]
    assert [y.requires_grad for y in ys] == [x.requires_grad or (w is not None and w.requires_grad) for x, w in zip(xs, ws)]
    live = [i for i in range(n) if ys[i].requires_grad]
    leaves = [i for i in live if xs[i].requires_grad]
    grads = torch.autograd.grad([ys[i] for i in live], [xs[i] for i in leaves] + each[:2], [gs[i] for i in live])
    for i in range(n):
        if xs[i].numel():
            nu.check_forward(f"y{i}", ys[i], xs[i], ws[i], EPS, at[i], f64(turns))
    for i, dx in zip(leaves, grads):
        if xs[i].numel():
            nu.check_dx(f"dx{i}", dx, xs[i], ws[i], gs[i], EPS, at[i], f64(turns))
    for k in (0, 1):
        nu.check_dw(f"dw{k}", grads[len(leaves) + k], [nu.dw_terms(xs[i], ws[i], gs[i], EPS, at[i], f64(turns)) for i in range(n) if of[i] == k and xs[i].numel()])


def test_only_wanted_gradients():
    turns, g = default_turns(64), rand(1, 2, 20, 64, seed=1)
    for x_wants, w_wants in ((True, False), (False, True)):
        x, w = rand(1, 2, 20, 64).requires_grad_(x_wants), weight(64).requires_grad_(w_wants)
        y = burst_norm_rotary(x, w, turns)
        (got,) = torch.autograd.grad(y, [x if x_wants else w], g)
        if x_wants:
            nu.check_dx("dx", got, x, w, g, EPS, np.arange(20)[None, None], f64(turns))
        else:
            nu.check_dw("dw", got, [nu.dw_terms(x, w, g, EPS, np.arange(20)[None, None], f64(turns))])
    with torch.no_grad():
        assert not burst_norm_rotary(x, w, turns).requires_grad
    xs = [rand(1, 2, 20, 64, seed=i).requires_grad_(True) for i in range(2)]      # only one of two results goes on
    w = weight(64).requires_grad_(True)
    dx, dw = torch.autograd.grad(burst_norm_rotary(xs, w, turns)[1], [xs[1], w], g)
    nu.check_dx("dx", dx, xs[1], w, g, EPS, np.arange(20)[None, None], f64(turns))
    nu.check_dw("dw", dw, [nu.dw_terms(xs[1], w, g, EPS, np.arange(20)[None, None], f64(turns))])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_zeros_and_rows_that_are_not_finite(dtype):
    x, g, w, turns = rand(1, 2, 12, 64, dtype=dtype), rand(1, 2, 12, 64, dtype=dtype, seed=1), weight(64), default_turns(64)
    x[0, 0, 3], x[0, 1, 5] = 0, 1e-30
    good = torch.ones(2, 12, dtype=torch.bool)
    bad = x.clone()
    bad[0, 0, 7, 9], bad[0, 1, 2, 0] = float("inf"), float("nan")
    good[0, 7] = good[1, 2] = False
    for v, keep in ((x, torch.ones_like(good)), (bad, good)):
        v = v.clone().requires_grad_(True)
        y = burst_norm_rotary(v, w, turns, 1e-5)
        (dx,) = torch.autograd.grad(y, v, g)
        one = burst_norm_rotary(x.clone().requires_grad_(True), w, turns, 1e-5)
        assert torch.equal(y[0][keep], one[0][keep])          # (other rows do not come in)
        assert bool(torch.isfinite(dx[0][keep]).all())
        if keep.all():
            at = np.arange(12)[None, None]
            nu.check_forward("y", y, v, w, 1e-5, at, f64(turns))
            nu.check_dx("dx", dx, v, w, g, 1e-5, at, f64(turns))


def test_errors():
    x, w, turns = rand(1, 2, 3, 64).requires_grad_(True), weight(64).requires_grad_(True), default_turns(64)
    for bad in (dict(weights=w[:63]), dict(weights=w.double()), dict(weights=w.bfloat16()), dict(weights=w.cpu()), dict(eps=0.0), dict(eps=float("nan")), dict(eps=-1.0),
                dict(turns=turns.float()), dict(positions=torch.zeros(4, dtype=torch.int64, device=DEV)), dict(x=rand(2, 3, 64)), dict(x=rand(1, 1, 2, 1)),
                dict(x=rand(1, 1, 2, 130), turns=None, weights=None)):
        with pytest.raises((ValueError, B.BurstError)):
            burst_norm_rotary(**dict(dict(x=x, weights=w, turns=turns), **bad))
    y = burst_norm_rotary(x, w, turns)
    with torch.no_grad():
        w.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = burst_norm_rotary(x, w, turns)
    y.sum().backward()
    with pytest.raises(RuntimeError, match="second time"):
        y.sum().backward()
    y = burst_norm_rotary(x, w, turns)
    dx, dw = torch.autograd.grad(y, [x, w], torch.ones_like(y), create_graph=True)
    plain = torch.autograd.grad(burst_norm_rotary(x, w, turns), [x, w], torch.ones_like(y))
    assert torch.equal(dx, plain[0]) and torch.equal(dw, plain[1]) and dx.requires_grad
    with pytest.raises(RuntimeError, match="gradients of its gradients"):
        dx.sum().backward()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            burst_norm_rotary(dual, w, turns)


def test_saved_tensors_come_back_elsewhere():
    x, w, turns, g = rand(1, 4, 30, 64).requires_grad_(True), weight(64).requires_grad_(True), default_turns(64), rand(1, 4, 30, 64, seed=1)
    want = torch.autograd.grad(burst_norm_rotary(x, w, turns), [x, w], g)
    elsewhere = lambda t: t.transpose(-1, 0).contiguous().transpose(-1, 0) if t.dim() > 1 else torch.stack([t, t], 1)[:, 0]   # noqa: E731
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: elsewhere(t.to(DEV))):
        y = burst_norm_rotary(x, w, turns)
    got = torch.autograd.grad(y, [x, w], g)
    assert torch.equal(got[0], want[0])
    assert torch.allclose(got[1], want[1], rtol=1e-5, atol=1e-5)   # (other granules, another order of sums)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[..., :-1] if t.dim() == 4 else t):
        y = burst_norm_rotary(x, w, turns)
    with pytest.raises(ValueError, match="sizes and device"):
        y.sum().backward()


def test_repeated_calls_streams_and_threads_of_two():
    x, w, turns, g = rand(2, 8, 700, 128, dtype=BF16).requires_grad_(True), weight(128, BF16).requires_grad_(True), default_turns(128), rand(2, 8, 700, 128, dtype=BF16, seed=1)
    y = burst_norm_rotary(x, w, turns)
    first = [y.detach(), *torch.autograd.grad(y, [x, w], g)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for s in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(s):
            y = burst_norm_rotary(x, w, turns)
            got.append([y.detach(), *torch.autograd.grad(y, [x, w], g)])
    torch.cuda.synchronize()
    for again in got:
        assert all(torch.equal(a, b) for a, b in zip(again, first))


def test_captured_pass_with_other_contents():
    x, w, g, turns = rand(1, 4, 100, 64, dtype=BF16), weight(64), rand(1, 4, 100, 64, dtype=BF16, seed=1), default_turns(64)

    def once():
        v, u = x.detach().requires_grad_(True), w.detach().requires_grad_(True)
        y = burst_norm_rotary(v, u, turns, EPS, 9)
        return [y.detach(), *torch.autograd.grad(y, [v, u], g)]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        once()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = once()
    for seed in (5, 6, 7):
        x.copy_(rand(1, 4, 100, 64, dtype=BF16, seed=seed))
        w.copy_(weight(64, seed=seed))
        graph.replay()
        want = once()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed


def test_captured_pass_beside_a_graph_of_the_same_leaves_that_lives():
    """The leaves' nodes are then the earlier graph's, on the default stream, which must not wait for a captured one: an error before it would, with
    nothing lost; when that graph is gone, passes are captured."""
    x, w, g = rand(1, 4, 100, 64, dtype=BF16).requires_grad_(True), weight(64).requires_grad_(True), rand(1, 4, 100, 64, dtype=BF16, seed=1)
    turns = default_turns(64)
    early = burst_norm_rotary(x, w, turns, EPS, 9)
    want = [early.detach(), *torch.autograd.grad(early, [x, w], g, retain_graph=True)]
    torch.cuda.synchronize()
    for wanted in ([x, w], [x], [w]):
        with pytest.raises(RuntimeError, match="captured backward pass"):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                torch.autograd.grad(burst_norm_rotary(x, w, turns, EPS, 9), wanted, g)
    torch.cuda.synchronize()
    again = torch.autograd.grad(early, [x, w], g)
    assert all(torch.equal(a, b) for a, b in zip(again, want[1:]))
    del early
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = burst_norm_rotary(x, w, turns, EPS, 9)
        out = [y.detach(), *torch.autograd.grad(y, [x, w], g)]
    for _ in range(3):
        for o in out:
            o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_c_entries_in_place_and_without_some_gradients():
    x, w, g, turns = rand(1, 3, 21, 64), weight(64), rand(1, 3, 21, 64, seed=1), default_turns(64)
    r = B.rotary(turns, amplitude=1.5)
    how = dict(pos=4 + np.arange(21)[None, None], turns=f64(turns), amplitude=1.5)
    y = x.clone()
    B.burst_norm_rotate([(y, y, None, 0, 4, None)], [(w, None)], EPS, r)
    nu.check_forward("y", y, x, w, EPS, **how)
    dx, dw = g.clone(), torch.empty_like(w)
    call = [(dx, dx, x, 0, 4, None)]
    ws = torch.empty(B.burst_norm_workspace_bytes(call, [(w, dw)], EPS, r), dtype=torch.uint8, device=DEV)
    B.burst_norm_rotate_bwd(call, [(w, dw)], EPS, r, ws)
    nu.check_dx("dx", dx, x, w, g, EPS, **how)
    nu.check_dw("dw", dw, [nu.dw_terms(x, w, g, EPS, **how)])
    again = torch.empty_like(dw)
    B.burst_norm_rotate_bwd([(g, None, x, 0, 4, None)], [(w, again)], EPS, r, ws)
    assert torch.equal(again, dw)
    only = torch.empty_like(x)
    B.burst_norm_rotate_bwd([(g, only, x, 0, 4, None)], [(w, None)], EPS, r)
    assert torch.equal(only, dx)
    with pytest.raises(B.BurstError):
        B.burst_norm_rotate_bwd(call, [(w, dw)], EPS, r, ws[:-4])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_with_norms(dtype):
    H, KV, d = 4, 2, 64
    leaves = [t.requires_grad_(True) for t in (rand(1, H, 50, d, dtype=dtype), rand(1, KV, 40, d, dtype=dtype, seed=1), rand(1, KV, 70, d, dtype=dtype, seed=2),
                                               weight(d), weight(d, seed=9))]
    q, k1, k2, wq, wk = leaves
    vs = [rand(1, KV, 40, d, dtype=dtype, seed=3), rand(1, KV, 70, d, dtype=dtype, seed=4)]
    g, turns = rand(1, H, 50, d, dtype=dtype, seed=5), default_turns(d)
    O, lse = burst_attention(q, [k1, k2], vs, causal=True, q_off=60, turns=turns, norms=(wq, wk), eps=1e-5)
    got = torch.autograd.grad(O, leaves, g)
    a, b, c = burst_norm_rotary([q, k1, k2], [wq, wk, wk], turns, 1e-5, offset=[60, 0, 40])
    O2, lse2 = burst_attention(a, [b, c], vs, causal=True, q_off=60)
    want = torch.autograd.grad(O2, leaves, g)
    assert torch.equal(O, O2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(got, want))
    f = [t.detach().double() for t in (q, k1, k2)]             # and without this package's norm
    n = [burst_rotary((x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.detach().double()).to(dtype), turns, o) for x, w, o in zip(f, (wq, wk, wk), (60, 0, 40))]
    O3, _ = burst_attention(n[0], n[1:], vs, causal=True, q_off=60)
    assert (O.float() - O3.float()).abs().max() <= (4e-2 if dtype == BF16 else 1e-4)
