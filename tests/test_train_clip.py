"""Norm of all gradients and their clipping, against 64 bits.  Squares are summed 32 numbers (16 of 32 bits) at a time in
32 bits, then in 64: below 2^-20 of the sum.  A clipped element is rounded twice in 32 bits at most (the factor, the
product) and once to its type."""
import math

import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, sp.BF16, 2.0 ** -8), "f16": (torch.float16, sp.F16, 2.0 ** -11),
         "f32": (torch.float32, sp.F32, 2.0 ** -24)}
EPS = 1e-6


class Case:
    def __init__(self, lengths, names, ranks=None, n_ranks=1, std=1e-2, shift=0, in_place=False, out=True):
        g = torch.Generator(device="cuda").manual_seed(len(lengths))
        self.names, self.n_ranks, self.ranks = names, n_ranks, ranks or [0] * len(lengths)
        self.buffers = [torch.zeros(n + 24, dtype=TYPES[t][0], device="cuda") for n, t in zip(lengths, names)]
        self.grads = [b[8 + shift:8 + shift + n] for b, n in zip(self.buffers, lengths)]
        for x in self.grads:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda") * std)
        self.around = [torch.full((n + 24,), 7.0, dtype=TYPES[t][0], device="cuda") for n, t in zip(lengths, names)]
        self.out = self.grads if in_place else [b[8:8 + n] for b, n in zip(self.around, lengths)] if out else None
        self.plan = sp.ClipPlan(lengths, [TYPES[t][1] for t in names], ranks=ranks, n_ranks=n_ranks)
        self.work = torch.empty(self.plan.workspace_bytes, dtype=torch.uint8, device="cuda")
        self.plan.set_workspace(self.work, self.work.numel())
        self.plan.set_tensors(self.grads, self.out)
        self.sums = torch.full((n_ranks,), 7.0, dtype=torch.float64, device="cuda")
        self.gathered = torch.empty(n_ranks, n_ranks, dtype=torch.float64, device="cuda")
        self.norms = torch.empty(n_ranks, 2, device="cuda")
        self.gather = sp.Plan(n_ranks, 8)

    def run(self, most=1.0, stream=None):
        self.plan.sums(self.sums, stream=stream)
        self.gather.allgather(self.sums, self.gathered, stream=stream)
        self.plan.scale(self.gathered, self.n_ranks, most, self.norms, eps=EPS, stream=stream)

    def check(self, before, most=1.0):
        each = [sum((x.double().square().sum().item() for x, r in zip(before, self.ranks) if r == i), 0.0) for i in range(self.n_ranks)]
        for got, want in zip(self.sums.tolist(), each):
            assert got == pytest.approx(want, rel=2.0 ** -20, abs=1e-300)
        norm = math.sqrt(sum(each))
        factor = 1.0 if norm == 0 else min(1.0, most / (norm + EPS))
        norm = torch.tensor(norm, dtype=torch.float64).float().item()  # beyond 32 bits' range an infinity, the factor not
        for n, f in self.norms.tolist():
            assert n == pytest.approx(norm, rel=2.0 ** -20, abs=1e-44) and f == pytest.approx(factor, rel=2.0 ** -20)
        if self.out is None:
            return
        for x, y, t in zip(before, self.out, self.names):
            want = x.double() * factor
            u, tiny = TYPES[t][2], {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}[t]
            assert ((y.double() - want).abs() <= (u + 2.0 ** -19) * want.abs() + tiny).all()
            if factor == 1.0:
                assert torch.equal(x, y)
        for b, y in zip(self.around, self.out):
            if y.data_ptr() != b[8:].data_ptr():
                continue
            assert (b[:8] == 7.0).all() and (b[8 + y.numel():] == 7.0).all()


MIXED = [100, 0, 1, 16384, 16385, 7, 100000, 33, 4096, 250001]


@pytest.mark.parametrize("n_ranks", [1, 3, 8, 40])
@pytest.mark.parametrize("std", [1e-2, 1e-6])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_tensors_of_all_types_and_ranks(n_ranks, std, shift):
    names = [("bf16", "f32", "f16")[i % 3] for i in range(len(MIXED))]
    c = Case(MIXED, names, [i * 7 % n_ranks for i in range(len(MIXED))], n_ranks, std=std, shift=shift)
    c.run()
    c.check(c.grads)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
def test_in_place(name):
    for std in (1e-1, 1e-6):
        c = Case(MIXED, [name] * len(MIXED), std=std, in_place=True)
        before = [x.clone() for x in c.grads]
        c.run()
        c.check(before)
        assert all((b[:8] == 0).all() and (b[8 + x.numel():] == 0).all() for b, x in zip(c.buffers, c.grads))


def test_the_norm_alone():
    c = Case([5000, 20], ["f32", "bf16"], out=False)
    before = [x.clone() for x in c.grads]
    c.run(0.5)
    c.check(before, 0.5)
    assert all(torch.equal(x, y) for x, y in zip(before, c.grads))


def test_numbers_whose_squares_32_bits_do_not_hold():
    for t, value in (("f32", 1e30), ("bf16", 1e37), ("f32", 1e-30), ("bf16", 1e-35), ("f32", 3e-42)):
        c = Case([3000, 40], [t, t])
        for x in c.grads:
            x.fill_(value)
        c.run()
        want = math.sqrt(3040) * c.grads[0][0].double().item()
        if want < 3e38:
            assert c.norms[0, 0].item() == pytest.approx(want, rel=1e-6, abs=2e-45)
        assert c.sums[0].item() == pytest.approx(want * want, rel=1e-6)
        c.check(c.grads)


def test_not_a_number_and_infinities():
    c = Case([3000, 4000], ["bf16", "f32"])
    c.grads[1][77] = float("nan")
    c.run()
    assert c.norms.isnan().all() and all(y.isnan().all() for y in c.out)
    c.grads[1][77] = float("inf")
    c.run()
    assert c.norms[0, 0] == float("inf") and c.norms[0, 1] == 0
    assert c.out[1][77].isnan() and (c.out[0] == 0).all() and (c.out[1][:77] == 0).all()


def test_zeros_and_nothing_allowed():
    c = Case([300], ["f32"], std=0.0)
    c.run(0.0)
    assert c.norms.tolist() == [[0.0, 1.0]] and (c.out[0] == 0).all()
    c = Case([300], ["f32"])
    c.run(0.0)
    assert c.norms[0, 1] == 0 and (c.out[0] == 0).all()
    c = Case([0, 0], ["f32", "bf16"], [0, 1], 2)
    c.run()
    assert (c.sums == 0).all() and c.norms.tolist() == [[0.0, 1.0]] * 2


def test_same_bits_when_replayed_and_other_tensors_after():
    c = Case([70000, 3, 20000], ["bf16", "f32", "f16"], [1, 0, 1], 2)
    c.run()
    torch.cuda.synchronize()
    want = [y.clone() for y in c.out], c.sums.clone()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        c.run(stream=stream)
    for _ in range(3):
        for y in c.out:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.sums, want[1]) and all(torch.equal(a, b) for a, b in zip(c.out, want[0]))
    others = [x.clone().mul_(2) for x in c.grads]
    c.plan.set_tensors(others, c.out)
    c.run()
    c.check(others)
