"""A wait of the scan that ran out belongs to its launch: later launches of the plan are whole, whether or not
the host has asked for the status in between.  (Only equality of bits and the status count here.)
"""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("direction", ["forward", "backward"])
def test_launches_after_one_that_gave_up_are_whole(direction):
    T, D = 200_000, 32    # a chain of 196 groups, far longer than a few looks at a word take
    g = torch.Generator(device="cuda").manual_seed(1)
    # the launches after it have inputs of their own: words that were left lying are not theirs
    inputs = []
    for _ in range(2):
        gate, x, dy = (torch.randn(T, D, generator=g, device="cuda") for _ in range(3))
        inputs.append((gate + 3, x, dy))

    def planned():
        plan = sp.ScanPlan([T], D, sp.F32)
        ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
        plan.set_workspace(ws, ws.numel())
        return plan

    plan, other = planned(), planned()
    carry = torch.empty(plan.carry_bytes // 4, device="cuda")

    def call(plan, which):
        gate, x, dy = inputs[which]
        out = torch.empty_like(x), torch.empty_like(x)
        if direction == "forward":
            plan.forward(gate, x, out[0])
            return out[:1]
        plan.backward(gate, x, carry, dy, *out)
        return out

    other.forward(*inputs[1][:2], torch.empty_like(inputs[1][0]), carry=carry)
    want = call(other, 1)
    assert other.status() == sp.OK
    call(plan, 0)
    assert plan.status() == sp.OK
    plan.set_wait_test(True, 5_000_000)
    call(plan, 0)
    plan.set_wait_test(False)
    later = [call(plan, 1), call(plan, 1)]
    assert plan.status() == sp.ERR_TIMEOUT    # of the launch that was withheld
    assert plan.status() == sp.OK
    for out in later:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
