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
