"""burst_cache_plan with parents that have no columns, or of no sequences: trees all the same, whose tokens hang on none; the torch call and the C entry."""
import numpy as np
import pytest
import torch

import plan_util
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.paged import burst_cache_plan

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x, *shape):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV).reshape(shape or np.asarray(x).shape)


@pytest.mark.parametrize("new,lengths,words,rows", [([3, 1, 70, 0, -1], [5, 0, 9, 40, 33], 1, 80), ([3, 1, 70, 0, -1], [5, 0, 9, 40, 33], 2, 80), ([900, 5, 2000], [0, 3, 9], 1, 3000),
                                                    ([], [], 1, 4)])
def test_parents_without_columns(new, lengths, words, rows):
    S, width, pages = len(new), 130, 400
    table = np.full((S, width), -1)
    want = plan_util.plan(new, lengths, table, list(range(pages)), pages, 16, rows, [[]] * S, words)
    for entry in ("torch", "C"):
        t, free, count = i32(table, S, width), i32(range(pages)), i32([pages])
        parents = torch.zeros(S, 0, dtype=torch.int32, device=DEV)
        if entry == "torch":
            got = burst_cache_plan(i32(new), i32(lengths), t, free, count, 16, rows, parents, words)
        else:
            got = [torch.full((n,), 77, dtype=torch.int32, device=DEV) for n in (S + 1, S)] + [torch.full((rows,), 77, dtype=torch.int64, device=DEV) for _ in range(2)]
            got.append(torch.full((rows, words), 77, dtype=torch.int64, device=DEV))
            B.burst_cache_plan(i32(new), i32(lengths), t, free, count, 16, *got[:4], parents, got[4])
        for name, g, w in zip(("starts", "lengths", "slots", "positions", "tree"), got, want):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w).reshape(g.shape)), (entry, name)
        assert np.array_equal(t.cpu().numpy(), want[5]) and count.tolist() == [want[7]], entry
