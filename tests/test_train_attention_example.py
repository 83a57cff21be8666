"""The training operators together, as a step divided over ranks uses them: norm, linear attention, clipping and the
allgathers between them, against the same layer on one rank in 64 bits."""
import math
import sys
from pathlib import Path

import pytest
import torch

import paper_2109_08751_b200 as sp

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))

pytestmark = pytest.mark.gpu


def layer(step, x, residual, dout, dr):
    """The layer token by token in 64 bits, and its gradients by torch's differentiation."""
    x = x.double().requires_grad_()
    w = {n: v.double().requires_grad_() for n, v in step.weights.items()}
    s = step.scale.double().requires_grad_()
    r = x + residual.double()
    u = r / (r.square().mean(1, keepdim=True) + 1e-6).sqrt() * s
    q, k, v = (t.unflatten(1, (step.heads, step.size)) for t in (u @ w["in"]).chunk(3, 1))
    decay, state, o = step.log_decay.double().exp()[:, None, None], 0.0, []
    for t in range(step.T):
        state = decay * state + k[t][:, :, None] * v[t][:, None]
        o.append(step.size ** -0.5 * (q[t][:, None] @ state)[:, 0])
    out = torch.stack(o).flatten(1) @ w["out"]
    ((out * dout.double()).sum() + (r * dr.double()).sum()).backward()
    return out.detach(), dict(x=x.grad, scale=s.grad, **{n: v.grad for n, v in w.items()})


@pytest.mark.parametrize("dtype,far", [(torch.float32, 1e-4), (torch.bfloat16, 4e-2), (torch.float16, 5e-3)])
def test_step_divided_over_ranks(dtype, far):
    # far: a dozen roundings of the type lie one behind another between x and a gradient, each at most half a step
    # (2^-8, 2^-11) of numbers that mix at random; 32 bits: 2^-24 of sums of some hundred numbers, and torch's products
    from sharded_attention_step import ShardedAttentionStep

    step = ShardedAttentionStep([70, 1, 130, 55], 64, 4, 32, dtype=dtype, most=0.5, seed=3)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, residual, dout, dr = (torch.randn(256, 64, generator=g, device="cuda").to(dtype) for _ in range(4))
    out, dx = step.gradients(x, residual, dout, dr)
    want, grads = layer(step, x, residual, dout, dr)
    step.status()
    got = dict(x=dx, scale=step.dscale, **step.grads)
    assert (out.double() - want).norm() <= far * want.norm()
    for n, v in grads.items():
        assert (got[n].double() - v).norm() <= far * v.norm(), n
    # clipped: one factor for all, from the norm of what was there
    before = {n: got[n].double().clone() for n in ("scale", "in", "out")}
    norm = math.sqrt(sum(v.square().sum().item() for v in before.values()))
    weights = {n: w.clone() for n, w in step.weights.items()}
    assert step.update().item() == pytest.approx(norm, rel=1e-5)
    u = torch.finfo(dtype).eps / 2
    for n, v in before.items():
        now = step.dscale if n == "scale" else step.grads[n]
        after = v * 0.5 / (norm + 1e-6)
        assert ((now.double() - after).abs() <= (u + 1e-5) * after.abs() + 2.0 ** -25).all(), n
    assert all(not torch.equal(weights[n], w) and w.isfinite().all() for n, w in step.weights.items())


def test_rows_gathered_in_8_bits():
    from sharded_attention_step import ShardedAttentionStep

    step = ShardedAttentionStep([16] * 4, 256, 2, 32)
    x = torch.randn(64, 256, device="cuda").bfloat16()
    y8, scales = step.share(x, 16)
    k = x.double()
    y = k / (k.square().mean(1, keepdim=True) + 1e-6).sqrt()
    for r in range(4):  # half a step of e4m3, or half of its smallest number times the scale
        each = scales[r].double().repeat_interleave(128, 1)
        assert ((y8[r].double() * each - y).abs() <= (2.0 ** -4 * y.abs()).maximum(2.0 ** -10 * each) * 1.001).all()


def test_the_whole_step_in_a_graph():
    from sharded_attention_step import ShardedAttentionStep

    step = ShardedAttentionStep([200, 56], 128, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, residual, dout = (torch.randn(256, 128, generator=g, device="cuda").bfloat16() for _ in range(3))
    step.gradients(x, residual, dout)
    torch.cuda.synchronize()
    want = [t.clone() for t in (step.dx, step.dscale, *step.grads.values())]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step.gradients(x, residual, dout)
        with torch.cuda.graph(graph, stream=stream):
            step.gradients(x, residual, dout)
    step.dx.zero_()
    graph.replay()
    torch.cuda.synchronize()
    step.status()
    assert all(torch.equal(a, b) for a, b in zip(want, (step.dx, step.dscale, *step.grads.values())))
    assert sp.OK == 0
