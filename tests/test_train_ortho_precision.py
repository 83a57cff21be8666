"""The orthogonalised update of bf16 matrices, as plans make it by themselves, against 64 bits: the result is at most
half as far off again as rounding to bf16 alone would leave it, at every size.

(One product of 11-bit operands is 2.5e-3 to 2.9e-3 off below 128 rows or columns, where rounding is 1.7e-3.)
"""
import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_ortho import far, matrices, planned, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["random", "lowrank", "decay"])
@pytest.mark.parametrize("rows,cols", [(3, 5), (16, 16), (32, 64), (64, 64), (64, 90), (90, 64), (80, 120), (64, 4096),
                                       (97, 140), (127, 127), (127, 190), (128, 128), (128, 256), (190, 128), (128, 4096),
                                       (256, 256), (300, 450), (1000, 700), (700, 2000)])
def test_bf16_results_are_as_good_as_rounded_ones(rows, cols, kind):
    for seed in range(4):
        u = matrices(1, rows, cols, kind, seed=seed).bfloat16()
        plan = planned(1, rows, cols, "bf16")
        out = torch.empty_like(u)
        plan.orthogonalize(u, out)
        assert plan.status() == sp.OK
        want = reference(u)
        assert far(out, want) <= 1.5 * far(want.bfloat16(), want)
