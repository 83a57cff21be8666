"""8-bit rows are y over the scale that is stored beside them: the quotient of two 32-bit numbers, rounded to e4m3 once.
With 32-bit rows y itself comes out too, so that the quotient can be formed here, to the bit."""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

EPS = 1e-6


def rows_and_8_bits(x, weight, block):
    rows, width = x.shape
    plan = sp.NormPlan(width, sp.F32, eps=EPS, block=block)
    y, y8 = torch.empty_like(x), torch.empty(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(rows, -(-width // block) if block else 1, device="cuda")
    plan.forward(rows, x, weight, y=y, y8=y8, scales=scales)
    return y, y8, scales


@pytest.mark.parametrize("rows,width,block", [(20000, 1024, 0), (40000, 512, 32), (3000, 5000, 128), (70001, 96, 64)])
def test_the_quotient_is_rounded_once(rows, width, block):
    g = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn(rows, width, generator=g, device="cuda")
    weight = torch.randn(width, generator=g, device="cuda")
    y, y8, scales = rows_and_8_bits(x, weight, block)
    # the scale is a quotient, too
    most = torch.stack([p.abs().amax(1) for p in y.split(block or width, 1)], 1)
    assert torch.equal(scales, most / torch.full_like(most, 448))  # torch multiplies by a plain number's inverse
    want = (y / scales.repeat_interleave(block or width, 1)[:, :width]).to(torch.float8_e4m3fn)
    assert int((want.view(torch.uint8) != y8.view(torch.uint8)).sum()) == 0


@pytest.mark.parametrize("size", [1e-29, 1e-20, 1e20, 1e37])
def test_quotients_of_rows_far_from_one(size):
    # the weights bring y to the ends of 32 bits' range; the smallest scales are 1e-30 / 448
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(4000, 256, generator=g, device="cuda")
    weight = torch.randn(256, generator=g, device="cuda") * size
    y, y8, scales = rows_and_8_bits(x, weight, 64)
    assert y.isfinite().all()
    want = (y / scales.repeat_interleave(64, 1)).to(torch.float8_e4m3fn)
    assert torch.equal(want.view(torch.uint8), y8.view(torch.uint8))


def test_quotients_of_infinities():
    # y / inf: 0 for finite numbers, NaN for infinite ones
    x = torch.randn(6, 128, device="cuda")
    weight = torch.ones(128, device="cuda")
    weight[70] = float("inf")
    y, y8, scales = rows_and_8_bits(x, weight, 64)
    assert scales[:, 0].isfinite().all() and scales[:, 1].isinf().all()
    assert y8[:, 70].float().isnan().all()
    rest = [i for i in range(64, 128) if i != 70]
    assert (y8[:, rest].float() == 0).all() and y8[:, :64].float().isfinite().all()
