"""burst_rotary as a node of torch's graph: tensors whose rows overlap in memory, forward mode, hooks on saved tensors, inputs that need no
gradient, several threads."""
import threading

import numpy as np
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paged_util import check_rotation, default_turns, f64
from paper_2403_09347_amd.autograd import burst_attention
from paper_2403_09347_amd.rotary import burst_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def rand(*shape, dtype=F32, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,strides", [((1, 2, 3, 8), (0, 60, 1, 1)), ((2, 1, 3, 8), (1, 60, 8, 1)), ((2, 2, 3, 8), (100, 1, 8, 1)),
                                           ((1, 2, 20, 8), (0, 60, 1, 1)), ((1, 1, 5, 128), (0, 0, 1, 1))])
def test_rows_that_overlap_in_memory(dtype, shape, strides):
    """Windows of a sequence, one element further each: a result that lay like them would have no unit stride along its rows."""
    base, g = rand(400, dtype=dtype), rand(400, dtype=dtype, seed=1).as_strided(shape, strides)
    x = base.as_strided(shape, strides)
    y = burst_rotary(x, default_turns(shape[3]), 3)
    check_rotation("y", y, x, 3 + np.arange(shape[2])[None, None], f64(default_turns(shape[3])))
    z = rand(*shape, dtype=dtype).requires_grad_(True)
    (dx,) = torch.autograd.grad(burst_rotary(z, default_turns(shape[3]), 3), z, g)
    check_rotation("dx", dx, g, 3 + np.arange(shape[2])[None, None], f64(default_turns(shape[3])), inverse=True)
