"""Captured backward passes of attention and of the rotation beside an eager graph of the same leaves that lives: an error, before the engine has the default stream
wait for the captured one; when that graph is gone, passes are captured and replayed."""
import pytest
import torch

from paged_util import default_turns
from paper_2403_09347_amd.autograd import burst_attention
from paper_2403_09347_amd.rotary import burst_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("how", ["plain", "turns", "norms", "rotation"])
def test_beside_a_graph_that_lives(how):
    leaves = [rand(1, h, n, 64, seed=h + n).requires_grad_(True) for h, n in ((4, 60), (2, 80), (2, 80))] + [(1 + rand(64, dtype=torch.float32, seed=s) / 8).requires_grad_(True) for s in (5, 6)]
    g = rand(1, 4, 60, 64, seed=9)
    turns = default_turns(64)                                  # (a copy from the host, which no capture has)
    of = {"plain": [0, 1, 2], "turns": [0, 1, 2], "norms": [0, 1, 2, 3, 4], "rotation": [0]}[how]

    def forward():
        if how == "rotation":
            return burst_rotary(leaves[0], turns, 9)
        q, k, v, wq, wk = leaves
        more = dict(turns=turns) if how != "plain" else {}
        if how == "norms":
            more.update(norms=(wq, wk))
        return burst_attention(q, [k], [v], causal=True, q_off=20, **more)[0]

    wanted = [leaves[i] for i in of]
    early = forward()
    want = [early.detach(), *torch.autograd.grad(early, wanted, g, retain_graph=True)]
    torch.cuda.synchronize()
    for some in [wanted] + [[w] for w in wanted]:
        with pytest.raises(RuntimeError, match="captured backward pass"):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                torch.autograd.grad(forward(), some, g)
    torch.cuda.synchronize()
    again = torch.autograd.grad(early, wanted, g)
    assert all(torch.equal(a, b) for a, b in zip(again, want[1:]))
    del early
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = forward()
        out = [y.detach(), *torch.autograd.grad(y, wanted, g)]
    for _ in range(3):
        for o in out:
            o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
