"""The orthogonalised update at the ends of its range: matrices of zeros, with any eps, give zeros, alone and beside
others; in a Muon step without gradient and momentum the weights move by their decay alone.

(Exact: zeros times finite numbers.  The decayed weight is one product and its rounding.)
"""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"f32": (sp.F32, torch.float32), "bf16": (sp.BF16, torch.bfloat16), "f16": (sp.F16, torch.float16)}


def planned(count, rows, cols, dtype, **kw):
    plan = sp.OrthoPlan(count, rows, cols, TYPES[dtype][0], **kw)
    ws = torch.full((plan.workspace_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
    plan.set_workspace(ws, ws.numel())
    return plan


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(70, 90), (130, 40)])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-30, 1e-20, 1e-18, 1e-7, 1.0])
def test_a_zero_matrix_gives_zeros(eps, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    u = (torch.randn(3, rows, cols, generator=g, device="cuda") * 1e-3).to(TYPES[dtype][1])
    whole, out = torch.empty_like(u), torch.empty_like(u)
    plan = planned(3, rows, cols, dtype, eps=eps)
    plan.orthogonalize(u, whole)
    u[1] = 0
    plan.orthogonalize(u, out)
    assert plan.status() == sp.OK
    assert (out[1] == 0).all()
    assert torch.equal(out[0], whole[0]) and torch.equal(out[2], whole[2])
    momentum = torch.zeros(3, rows, cols, device="cuda")
    weight = torch.randn(3, rows, cols, generator=g, device="cuda")
    moved = torch.empty_like(weight)
    plan.muon_step(u, momentum, momentum, weight, moved, weight_dtype=sp.F32, lr=0.25, weight_decay=0.5)
    assert plan.status() == sp.OK
    assert torch.equal(moved[1], weight[1] * 0.875)
    assert torch.isfinite(moved).all() and (momentum[1] == 0).all()
