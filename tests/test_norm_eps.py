"""What eps a norm takes: 2^-126 and more (smaller ones have no root on the device: rows of zeros would come back as NaN), finite."""
import ctypes

import pytest
import torch

from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.rotary import burst_norm_rotary
from test_norm_refusals import back, call, norm_rows, store
from test_paged_refusals import E_NULL, E_SHAPE, paged

LEAST = 2.0 ** -126


@pytest.mark.parametrize("eps", [0.0, -0.0, -1e-6, 1e-45, 1e-40, 1.17e-38, float("inf"), float("-inf"), float("nan")])
def test_refused(eps):
    assert call(norm_rows(), eps=eps) == E_SHAPE and back(norm_rows(frm=12288), eps=eps) == E_SHAPE
    for name in ("q_weight", "k_weight"):
        assert store(paged(), B.BurstStore(eps=eps, **{name: 4096})) == E_SHAPE


@pytest.mark.parametrize("eps", [LEAST, 1e-6, 1.0, 3e38])
def test_taken(eps):
    """Refused for something that is looked at later."""
    assert call(norm_rows(y=None), eps=eps) == E_NULL and back(norm_rows(), eps=eps) == E_NULL
    assert store(paged(starts=None), B.BurstStore(eps=eps, k_weight=4096)) == E_NULL
    w = B.BurstNormWeight(w=4096, dw=8192)
    assert B.load().burst_norm_workspace_bytes(ctypes.byref(norm_rows(frm=12288)), 1, ctypes.byref(w), 1, eps, None, 64, 0) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_zeros_with_the_least(dtype):
    x = torch.zeros(1, 1, 3, 64, dtype=dtype, device="cuda:0")
    x[0, 0, 1] = 1
    assert bool((burst_norm_rotary(x, None, None, LEAST) == x).all())
    for eps in (LEAST * 0.99, 1e-45, 1e-50):
        with pytest.raises(ValueError, match="eps"):
            burst_norm_rotary(x, None, None, eps)
