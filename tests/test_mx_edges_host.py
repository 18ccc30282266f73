"""MXFP4 rows and the calls around them at the edges of what they take, without a GPU."""
import numpy as np
import pytest
import torch

from paper_2508_05700_amd import binding as b


def test_sizes_are_remembered_by_the_number():
    # (a tensor of one number is a number too, and may hold another one later)
    n = torch.tensor(64)
    assert b.emb_row_bytes(n, "mxfp4") == 48 and b.emb_cache_index_bytes(n) == 16
    n.fill_(128)
    assert b.emb_row_bytes(n, "mxfp4") == 80 and b.emb_cache_index_bytes(n) == 32
    assert b.emb_row_bytes(np.int32(96), "mxfp4") == 64 == b.emb_row_bytes(96, "mxfp4")
    with pytest.raises(b.EmbError):
        b.emb_cache_index_bytes(-1)
