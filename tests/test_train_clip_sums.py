"""Sums of squares are 64-bit sums: the square of a 32-bit number is held exactly, and an addition of n of them, in whatever
order, is off by at most n 2^-53 of a sum of numbers that are never negative."""
import pytest
import torch

from test_train_clip import Case

pytestmark = pytest.mark.gpu


def want_of(c):
    # sums of some thousand squares each, then of those: 64-bit additions, as far off as the ones they are compared with
    return [sum((x.double().square().sum().item() for x, r in zip(c.grads, c.ranks) if r == i), 0.0) for i in range(c.n_ranks)]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("value", [0.1, 0.0013, 3.0])
def test_equal_numbers(name, value):
    # all groups of squares round alike: what is lost in 32 bits adds up
    c = Case([1 << 18, 77777, 5], [name] * 3)
    for x in c.grads:
        x.fill_(value)
    c.plan.sums(c.sums)
    n = sum(x.numel() for x in c.grads)
    assert c.sums[0].item() == pytest.approx(c.grads[0][0].double().item() ** 2 * n, rel=n * 2.0 ** -53)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shift", [0, 3])
def test_numbers_of_many_sizes(name, shift):
    # sizes of 1e-4 to 1e2 beside one another, ranks of their own, odd lengths
    c = Case([1 << 17, 50001, 3, 33333], [name] * 4, [2, 0, 2, 1], 3, shift=shift)
    g = torch.Generator(device="cuda").manual_seed(7)
    for x in c.grads:
        x.mul_((10 ** (torch.rand(x.shape, generator=g, device="cuda") * 6)).to(x.dtype))
    c.plan.sums(c.sums)
    for got, want in zip(c.sums.tolist(), want_of(c)):
        assert got == pytest.approx(want, rel=2 * (1 << 18) * 2.0 ** -53)
