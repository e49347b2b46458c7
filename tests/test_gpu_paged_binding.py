"""The binding's calls of the rotation and the paged cache on the device: against the torch calls, bit for bit, and what the library refuses."""
import pytest
import torch

from paged_util import Batch, default_turns
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention
from paper_2403_09347_amd.rotary import burst_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotate(dtype):
    base = torch.randn(2, 50, 4, 64, device=DEV).to(dtype)
    turns = default_turns(64)
    at = torch.randint(0, 1 << 20, (2, 50), device=DEV)
    xs = [base.transpose(1, 2), base.transpose(1, 2).contiguous(), base.transpose(1, 2)[:, :1].expand(2, 4, 50, 64)]
    ys = [torch.empty(2, 4, 50, 64, dtype=dtype, device=DEV) for _ in xs]
    B.burst_rotate(xs, ys, B.rotary(turns), offsets=[5, 0, 9], positions=[at, None, at[:1].expand(2, 50)])
    want = burst_rotary(xs, turns, [5, 0, 9], [at, None, at[0]])
    assert all(torch.equal(y, w) for y, w in zip(ys, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pool", ["head", "seq"])
def test_append_and_attend(dtype, pool):
    b = Batch([100, 40, 7], [30, 1, 2], 4, 2, 64, dtype=dtype, pool=pool, packed=True)
    turns, r = default_turns(64), B.rotary(default_turns(64))            # (the blocks keep what they were made from)
    p = B.paged_params(33, 4, 2, 64, dtype, b.k_pages, b.table.clone(), b.lengths.clone(), b.starts.clone(), b.scale, full_p=True)
    p.q_strides[:], p.kv_strides[:] = b.q.stride()[:2], b.k.stride()[:2]
    pages = b.k_pages.clone(), b.v_pages.clone()
    want = burst_cache_append(b.k, b.v, *pages, b.table, b.lengths, b.starts, q=b.q, turns=turns)
    q = torch.empty(33, 4, 64, dtype=dtype, device=DEV)
    B.burst_cache_append(b.k, b.v, b.k_pages, b.v_pages, b.q, q, None, r, p)
    assert torch.equal(q, want) and torch.equal(b.k_pages, pages[0]) and torch.equal(b.v_pages, pages[1])
    with pytest.raises(B.BurstError):
        B.burst_cache_append(b.k, b.v, b.k_pages, b.v_pages, b.q, None, None, r, p)
    p.q_strides[:] = [0, 0]
    O, lse = torch.empty_like(q), torch.empty(33, 4, device=DEV)
    ws = torch.empty(B.burst_paged_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    B.burst_paged_fwd(q, b.k_pages, b.v_pages, O, lse, p, ws)
    got = burst_paged_attention(q, *b.args(), full_p=True)
    assert torch.equal(O, got[0]) and torch.equal(lse, got[1])
