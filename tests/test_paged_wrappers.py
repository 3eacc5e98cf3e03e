"""What the allocating wrapper of the paged attention asks for, without a GPU: nothing is enqueued."""
import pytest
import torch

import paper_2310_01889_amd as ra


def test_offsets_need_their_bound():
    """Row offsets without max_new would leave all but a request's first row at zero, as padding is."""
    bf, i32 = torch.bfloat16, torch.int32
    q, pages = torch.zeros(5, 2, 64, dtype=bf), torch.zeros(3, 16, 1, 64, dtype=bf)
    table, lens, cu = torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(ValueError, match="max_new"):
        ra.paged_attention(q, pages, pages, table, lens, cu)
