"""The factor at the ends of its range, as documented: nothing to clip (a norm of 0, or any number allowed) is factor 1."""
import pytest
import torch

from test_train_clip import Case

pytestmark = pytest.mark.gpu

INF = float("inf")


def test_any_number_allowed():
    c = Case([3000, 40], ["bf16", "f32"], [0, 1], 2, std=1e3)
    c.run(INF)
    c.check(c.grads, INF)
    assert (c.norms[:, 1] == 1).all() and all(torch.equal(x, y) for x, y in zip(c.grads, c.out))
    c.grads[1][7] = INF
    c.run(INF)
    assert (c.norms == torch.tensor([INF, 1.0], device="cuda")).all() and all(torch.equal(x, y) for x, y in zip(c.grads, c.out))
    c.grads[1][7] = float("nan")
    c.run(INF)
    assert c.norms.isnan().all() and all(y.isnan().all() for y in c.out)


@pytest.mark.parametrize("most", [0.0, 1e-9, 1.0])
def test_a_norm_of_zero(most):
    c = Case([300], ["f32"], std=0.0)
    c.run(most)
    c.check(c.grads, most)
    assert c.norms.tolist() == [[0.0, 1.0]]
