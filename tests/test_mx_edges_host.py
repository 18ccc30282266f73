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


F32, BF16, INT8, MX = 0, 1, 2, 6
FAKE = 0x1000   # a non-null, aligned address
OK, UNSUPPORTED, HIP = 0, -2, -4
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="launches, which only fail where there is no GPU")


def test_product_of_more_rows_than_it_takes_is_refused():
    f = b.lib().emb_rows_product
    most = (1 << 31) - 2048
    for M, N in ((1, most + 1), (most + 1, 1), (1, 1 << 31), (33, 1 << 40)):
        for x in (F32, BF16, MX):
            assert f(FAKE, x, 32, M, FAKE, N, 32, FAKE, BF16, N, None) == UNSUPPORTED


@no_gpu
def test_product_of_more_threads_than_a_grid_holds_is_launched():
    # (what fails is the launch, for want of a GPU: none of these sizes is refused)
    f = b.lib().emb_rows_product
    most = (1 << 31) - 2048
    for x in (F32, BF16, MX):
        for M, N, D in ((33, 730_000_000, 32), (48, most, 32), (1, most, 32), (32, most, 32), (64, most, 32), (most, 1, 32), (most, 64, 32),
                        (17, 1_100_000_000, 256), (200, 600_000_000, 32)):
            assert f(FAKE, x, D, M, FAKE, N, D, FAKE, BF16, N, None) == HIP, (x, M, N, D)
