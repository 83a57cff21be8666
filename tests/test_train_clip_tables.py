"""What set_tensors says holds for calls that were captured before it, too."""
import pytest
import torch

from test_train_clip import Case

pytestmark = pytest.mark.gpu


def captured(c):
    c.run()  # the collective's first launch allocates
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        c.run(stream=stream)
    return graph


def test_captured_with_outputs_and_replayed_without():
    c = Case([70000, 3, 0, 20000], ["bf16", "f32", "f16", "f16"], [1, 0, 1, 1], 2)
    graph = captured(c)
    want = c.norms.clone()
    c.plan.set_tensors(c.grads)
    for y in c.out:
        y.fill_(3.0)
    before = [x.clone() for x in c.grads]
    c.norms.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.norms, want) and want[0, 1] < 1
    assert all((y == 3.0).all() for y in c.out) and all(torch.equal(x, y) for x, y in zip(before, c.grads))


def test_captured_without_outputs_and_replayed_with():
    c = Case([70000, 3, 20000], ["bf16", "f32", "f16"], [1, 0, 1], 2, out=False)
    graph = captured(c)
    c.out = [torch.zeros_like(x) for x in c.grads]
    c.plan.set_tensors(c.grads, c.out)
    graph.replay()
    torch.cuda.synchronize()
    assert c.norms[0, 1] < 1
    c.check(c.grads)


def test_captured_out_of_place_and_replayed_in_place():
    c = Case([70000, 3, 20000], ["bf16", "f32", "f16"], [1, 0, 1], 2)
    graph = captured(c)
    before = [x.clone() for x in c.grads]
    for y in c.out:
        y.fill_(3.0)
    c.plan.set_tensors(c.grads, c.grads)
    graph.replay()
    torch.cuda.synchronize()
    assert all((y == 3.0).all() for y in c.out)
    c.out = c.grads
    c.check(before)
