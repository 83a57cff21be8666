"""A router whose chosen weights are divided by their sum, with one choice (or one that can be made): the weight is 1,
exactly, and no gradient of it reaches the logits, where a weight of 1 - 2^-23 would leave 1e-7 of it beside the far
smaller gradient of the balance loss."""
import pytest
import torch

from test_train_router import TYPES, logits_of, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E", [1, 15, 64, 200, 700])
def test_one_choice(E, dtype):
    l = logits_of(400, E, dtype, E)
    got = run(l, [400], 1, True, dtype)
    assert (got["wgt"] == 1).all()
    without = run(l, [400], 1, True, dtype, dw=False)
    assert torch.equal(got["d"], without["d"])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_one_expert_left_of_more_choices(dtype):
    l = logits_of(60, 20, dtype, 3)
    left = torch.arange(60) % 20
    masked = torch.full_like(l, float("-inf"))
    masked[torch.arange(60), left] = l[torch.arange(60), left]
    got = run(masked, [60], 4, True, dtype)
    assert (got["wgt"][:, 0] == 1).all() and (got["wgt"][:, 1:] == 0).all()
    assert torch.equal(got["d"], run(masked, [60], 4, True, dtype, dw=False)["d"])
