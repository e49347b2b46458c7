"""What the paged calls write, as torch sees it: versions of the tensors written, and tensors that want a gradient."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paged_util import Batch, default_turns
from paper_2403_09347_amd.autograd import burst_attention
from paper_2403_09347_amd.harness import PagedWalk
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def append(b, **kw):
    return burst_cache_append(b.k, b.v, *b.args(), **kw)


def attend(b, **kw):
    return burst_paged_attention(b.q, *b.args(), **kw)


def test_forward_mode_is_refused():
    b = Batch([40, 20], [3, 1], 4, 2, 64)
    t = dict(k=b.k, v=b.v, k_pages=b.k_pages, v_pages=b.v_pages, table=b.table, lengths=b.lengths, starts=b.starts, q=b.q, turns=default_turns(64))
    with fwd.dual_level():
        dual = {n: fwd.make_dual(t[n].clone(), torch.ones_like(t[n])) for n in ("k", "v", "k_pages", "v_pages", "q")}
        for n in dual:
            with pytest.raises(RuntimeError, match="forward-mode"):
                burst_cache_append(**dict(t, **{n: dual[n]}))
        a = dict(q=b.q, **{n: t[n] for n in ("k_pages", "v_pages", "table", "lengths", "starts")})
        for n in ("k_pages", "v_pages", "q"):
            with pytest.raises(RuntimeError, match="forward-mode"), torch.no_grad():
                burst_paged_attention(**dict(a, **{n: dual[n]}))
        for n, like in (("out", b.q.contiguous()), ("lse", torch.empty(4, 4, device=DEV))):
            with pytest.raises(RuntimeError, match="forward-mode"):
                burst_paged_attention(**a, **{n: fwd.make_dual(like, like.clone())})
        with pytest.raises(RuntimeError, match="forward-mode"):
            PagedWalk(b.k_pages, b.v_pages, 0.125).step(dual["q"], b.k, b.v, b.table, b.lengths, b.starts)


def test_written_tensors_have_another_version():
    b = Batch([40, 20], [3, 1], 4, 2, 64)
    before = b.k_pages._version, b.v_pages._version, b.k._version, b.q._version
    append(b, q=b.q, turns=default_turns(64))
    after = b.k_pages._version, b.v_pages._version, b.k._version, b.q._version
    assert after[0] > before[0] and after[1] > before[1] and after[2:] == before[2:]
    out, lse = torch.empty_like(b.q.contiguous()), torch.empty(4, 4, device=DEV)
    versions = out._version, lse._version, b.k_pages._version, b.v_pages._version
    attend(b, out=out, lse=lse)
    assert out._version > versions[0] and lse._version > versions[1] and (b.k_pages._version, b.v_pages._version) == versions[2:]


def test_a_graph_that_saved_the_pool_does_not_use_what_was_written_since():
    """A walk over a chunk that lies in the pool, its backward after the next token was appended."""
    pool = [torch.randn(4, 2, 64, 64, device=DEV).to(BF16) for _ in range(2)]
    q = torch.randn(1, 4, 10, 64, device=DEV).to(BF16).requires_grad_(True)
    table, lengths = torch.arange(4, dtype=torch.int32, device=DEV).view(1, 4), torch.tensor([200], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    new = torch.randn(1, 2, 64, device=DEV).to(BF16)
    for i in range(2):
        O, _ = burst_attention(q, pool[0][:1], pool[1][:1])
        if i:
            burst_cache_append(new, new, *pool, table, lengths, starts)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                O.sum().backward()
        else:
            O.sum().backward()
    O, _ = burst_attention(q, pool[0][:1], pool[1][:1])
    out = q.detach().new_empty(10, 4, 64)
    y = (q[0].transpose(0, 1) * out).sum()                    # saves out
    burst_paged_attention(q.detach()[0].transpose(0, 1), *pool, table, lengths, torch.tensor([0, 10], dtype=torch.int32, device=DEV), out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_inference_mode():
    with torch.inference_mode():
        b = Batch([40, 20], [3, 1], 4, 2, 64)
        append(b)
        want = attend(b)
    append(b)                                                 # such tensors have no version, and cannot be saved
    got = attend(b)
    assert torch.equal(want[0], got[0])
    c = Batch([40, 20], [3, 1], 4, 2, 64)
    with torch.inference_mode():
        append(c)
        got = attend(c)
    assert torch.equal(want[0], got[0])


def test_pages_that_want_a_gradient_are_refused():
    b = Batch([40, 20], [3, 1], 4, 2, 64)
    wants = lambda t: t.clone().requires_grad_(True)          # noqa: E731
    plain = (b.table, b.lengths, b.starts)
    for k, v in ((wants(b.k_pages), b.v_pages), (b.k_pages, wants(b.v_pages))):
        with pytest.raises(ValueError, match="gradient"):
            burst_paged_attention(b.q, k, v, *plain)
        with pytest.raises(ValueError, match="gradient"):
            burst_cache_append(b.k, b.v, k, v, *plain)
        with torch.no_grad():
            O, _ = burst_paged_attention(b.q, k, v, *plain)
            assert torch.equal(O, attend(b)[0])
    lse = torch.empty(4, 4, device=DEV)
    with pytest.raises(ValueError, match="gradient"):
        attend(b, lse=wants(lse))
    with pytest.raises(ValueError, match="gradient"):
        attend(b, out=wants(b.q.contiguous()))
