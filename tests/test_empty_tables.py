"""Tables without sequences, whatever strides they have (numpy's and torch's empty matrices have any), make a parameter block."""
import numpy as np
import torch

from paper_2403_09347_amd import binding as B


def test_a_block_of_no_sequences():
    pages = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)        # noqa: E731
    for table in (i32(np.full((0, 5), -1)), torch.empty_strided((0, 5), (0, 3), dtype=torch.int32), torch.zeros(0, 5, dtype=torch.int32)):
        p = B.paged_params(4, 4, 2, 64, torch.bfloat16, pages, table, i32([]), i32([0]))
        assert (p.sequences, p.width, p.table_stride) == (0, 5, 0)
