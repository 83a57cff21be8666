"""Calls of the orthogonalised update that follow one another without a pause: CTA pairs leave and others take
their place on the same SMs all the time, and every call has to give the bits of the first.

The results themselves are compared with the formulas elsewhere; here only equality counts.
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
@pytest.mark.parametrize("count,rows,cols", [(1, 40, 40), (4, 256, 256), (3, 300, 100), (80, 64, 64)])
def test_calls_back_to_back_repeat_their_bits(count, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    u = (torch.randn(count, rows, cols, generator=g, device="cuda") * 1e-3).to(TYPES[dtype][1])
    plan = planned(count, rows, cols, dtype)
    outs = [torch.empty_like(u) for _ in range(24)]
    for out in outs:
        plan.orthogonalize(u, out)
    assert plan.status() == sp.OK
    assert torch.isfinite(outs[0]).all()
    assert all(torch.equal(outs[0], out) for out in outs[1:])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("count,rows,cols", [(1, 40, 40), (3, 300, 1000), (80, 200, 200)])
def test_waits_that_run_out_are_reported(count, rows, cols, dtype):
    """Finished products are withheld on purpose, with one tile a CTA pair and with several: every kernel gives
    up after the limit, the plan says so, and works again afterwards."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    u = (torch.randn(count, rows, cols, generator=g, device="cuda") * 1e-3).to(TYPES[dtype][1])
    plan = planned(count, rows, cols, dtype, steps=1)
    first, again = torch.empty_like(u), torch.empty_like(u)
    plan.orthogonalize(u, first)
    assert plan.status() == sp.OK
    plan.set_wait_test(True, 5_000_000)
    plan.orthogonalize(u, again)
    assert plan.status() == sp.ERR_TIMEOUT
    plan.set_wait_test(False)
    plan.orthogonalize(u, again)
    assert plan.status() == sp.OK and torch.equal(first, again)
