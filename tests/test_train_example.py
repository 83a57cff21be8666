"""The example that runs the training operators together (examples/sharded_training_step.py) against the
same model in 64 bits with torch's own differentiation, whole instead of divided.

Tolerance: everything is in 32 bits; the products with the weights are sums of at most 96 terms and the
recurrence keeps at most about 60 steps' worth of rounding, so gradients are good to 1e-4 of their norm.
The update is the orthogonalised gradient, whose steps magnify a relative error of the gradient in the
small singular values by up to 3.4445 ** 5 / 3.4445 = 141: 1.5e-2 of the update's norm.
"""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
spec = importlib.util.spec_from_file_location(
    "sharded_training_step", Path(__file__).resolve().parent.parent / "examples" / "sharded_training_step.py")
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


@pytest.mark.parametrize("tokens", [[50, 50], [13, 0, 64, 1], [40]], ids=str)
def test_step_equals_the_undivided_model(tokens):
    width, channels, experts, k = 64, 96, 12, 3
    step = example.ShardedStep(tokens, width, channels, experts, k, dtype=torch.float32)
    T = sum(tokens)
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(T, width, generator=g, device="cuda")
    dchosen = torch.randn(T, k, generator=g, device="cuda") * 0.1
    before = {n: w.clone() for n, w in step.weights.items()}
    loss, grads = step.run(h, dchosen)
    step.status()

    w = {n: v.double().requires_grad_() for n, v in before.items()}
    gx = h.double() @ w["in"]
    a = torch.sigmoid(gx[:, :channels])
    b = torch.sigmoid(-gx[:, :channels]) * gx[:, channels:]
    state, ys = torch.zeros(channels, dtype=torch.float64, device="cuda"), []
    for t in range(T):
        state = a[t] * state + b[t]
        ys.append(state)
    logits = torch.stack(ys) @ w["router"]
    p = torch.softmax(logits, 1)
    idx = step.indices.long()
    assert torch.equal(idx, torch.topk(p, k, 1).indices)
    chosen = p.gather(1, idx)
    chosen = chosen / chosen.sum(1, keepdim=True)
    f = torch.bincount(idx.reshape(-1), minlength=experts).double() / (T * k)
    want = (step.alpha * experts * (p.mean(0) * f).sum()
            + step.beta * (torch.logsumexp(logits, 1) ** 2).mean())
    (want + (dchosen.double() * chosen).sum()).backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * abs(want.item())
    for n in w:
        err = (grads[n].double() - w[n].grad).norm() / w[n].grad.norm()
        assert err.item() <= 1e-4, (n, err)
        u = w[n].grad * (1 + 0.95)   # first step: momentum = gradient, Nesterov's look ahead
        x = u / u.norm()
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        for _ in range(5):
            q = x @ x.T
            x = 3.4445 * x + (-4.7750 * q + 2.0315 * (q @ q)) @ x
        x = x.T if tall else x
        move = step.lr * 0.2 * math.sqrt(max(x.shape)) * x
        moved = (1 - step.lr * 0.01) * before[n].double() - step.weights[n].double()
        assert ((moved - move).norm() / move.norm()).item() <= 1.5e-2, n


def test_steps_balance_the_experts():
    """With only the balance loss to follow, the loss falls."""
    tokens = [256, 256]
    step = example.ShardedStep(tokens, 64, 64, 8, 2, dtype=torch.bfloat16, alpha=1.0, beta=0.0, lr=0.01)
    g = torch.Generator(device="cuda").manual_seed(3)
    h = (torch.randn(512, 64, generator=g, device="cuda") + 0.5).bfloat16()
    zero = torch.zeros(512, 2, device="cuda")
    losses = [step.run(h, zero)[0].item() for _ in range(30)]
    step.status()
    assert losses[-1] < losses[0]
    assert abs(losses[-1] - 1.0) < abs(losses[0] - 1.0)   # 1: every expert gets the same
