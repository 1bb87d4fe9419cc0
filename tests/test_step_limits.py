"""Sizes at which the calls around the products begin to refuse, from the tiles and workgroups that they launch (no GPU needed; 256 compute units)."""
import pytest
import torch

import paper_2402_17985_amd as fq
from tests.test_step_api import HIP, RANGE, product

SIDE = 2**31 - 257


def sizes(M, N, K=64, group=64):
    return product(M=M, N=N, K=K, ldx=K, ldy=N, group=group, x_dtype=fq.FQ_BF16)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N", [(524288, 4096), (200000, 11008), (67105, 32000), (16737, 128256), (2**30 - 64, 63), (49, 2**31 - 2**20), (32, 2**27 - 1), (1, SIDE), (2**17, 2**20 - 256)])
def test_products_of_many_outputs_are_not_refused(M, N, group):
    """They reach the launch, which fails where there is no GPU."""
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU: reaching the launch is what comes back as an error")
    assert sizes(M, N, group=group) == HIP


@pytest.mark.parametrize("M,N,K,group", [(SIDE + 1, 8, 64, 64), (SIDE, 63, 64, 64), (8, SIDE + 1, 64, 64), (64 * 2**20, 256 * 16, 64, 128), (64 * 2**20, 128 * 16, 64, 32), (48, 2**28, 64, 64),
                                         (32, 2**29, 64, 32), (16, 2**27, 8192, 64), (2**31 - 1, 2**31 - 1, 64, 64)])
def test_products_that_no_launch_holds_are_refused(M, N, K, group):
    """2^32 threads: tiles of 64 x 256, of 64 x 128 and four waves, of 48 x 64, 32 x 128 and 16 x 32 and sixteen; a side that 31 bits do not hold with the last tile filled up."""
    assert sizes(M, N, K, group) == RANGE
