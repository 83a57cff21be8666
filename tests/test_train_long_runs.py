"""Sizes at which a CTA goes on: clipping with more chunks than CTAs, whose runs hold many chunks of a tensor and ranks that
change in their middle, and the norm of rows so wide that one is a CTA's, with many rows a CTA."""
import pytest
import torch

import test_train_norm
from test_train_clip import Case

pytestmark = pytest.mark.gpu

# 1400 chunks of 16384 elements and some: more than two for each of 592 CTAs
LENGTHS = [9000000, 1, 16384, 700001, 33, 0, 5000003, 2000, 1048576, 7, 4100000, 999, 16385, 3000000, 12, 65536]


@pytest.mark.parametrize("n_ranks", [1, 3, 7])
@pytest.mark.parametrize("in_place", [False, True])
def test_clipping_with_runs_of_many_chunks(n_ranks, in_place):
    names = [("bf16", "f32", "f16", "bf16")[i % 4] for i in range(len(LENGTHS))]
    c = Case(LENGTHS, names, [i * 5 % n_ranks for i in range(len(LENGTHS))], n_ranks, std=0.3, shift=1, in_place=in_place)
    before = [x.clone() for x in c.grads]
    c.run()
    c.check(before)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", [(700, 8200), (500, 12288), (500, 16390), (450, 20000), (470, 32768), (451, 32767)])
def test_wide_rows_with_many_rows_a_cta(rows, width, name):
    test_train_norm.test_forward_and_backward(rows, width, 0, 0, name)
