"""Sizes of single tokens that the library refuses reach it, whatever the scale, no GPU."""
import pytest

import paper_2109_08751_b200 as sp
from test_train_host import GPU_SIZED, refused

A = [GPU_SIZED * (i + 1) for i in range(8)]


@pytest.mark.parametrize("size", [0, -1, -4])
@pytest.mark.parametrize("scale", [None, 0.5])
def test_no_keys(size, scale):
    refused(sp.ERR_ARG, sp.linear_attention_step, 3, 2, size, 32, sp.BF16, A[0], A[1], A[2], A[3], A[4], A[4], A[5], scale=scale,
            q_ld=128, k_ld=128)
    refused(sp.ERR_ARG, sp.LinearAttentionPlan, [4], 2, size, 64, scale=scale)
