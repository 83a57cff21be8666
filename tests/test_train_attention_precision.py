"""How far linear attention is off as a whole, beside the limits for each number of test_train_attention.

States: one chunk adds 32 products to a sum of 32 bits (8 steps of 16 tokens for each of bf16's four parts), of which each
rounds off half a last bit, 2^-24 of a sum that has grown to half of its final size on average: in random directions
sqrt(32) 2^-25 = 2^-22.5.  A weight is an exponential that is 2^-22 off at most (two last bits) and mostly 2^-24, and the same goes
for the decay of each of up to 9 chunks.  Together below 2^-20 of the state's norm.  A lost part would be seen: the
fourth of bf16's and what the third of a weight's numbers adds hold 2^-18 at most, 2^-19 in the mean (checked here), the second of
fp16's 2^-12.

Outputs of 16 bits: their own rounding leaves their norm r off (computed here).  Every token's part is rounded once more on
the way, as a weight (tokens of the chunk) or with the state (tokens before it), which of sums of random numbers leaves r
again: sqrt(2) r together.  1.5 r leaves the rest of it, a sixteenth, to 32-bit arithmetic and to chance.  Outputs of 32 bits:
sums of some hundred numbers in two steps, 2^-21."""
import pytest
import torch

from test_train_attention import Case

DECAYS = [1 - 2.0 ** -5.5, 1 - 2.0 ** -10, 0.3]  # no powers of two, nor is the scale, which against time multiplies c


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kd,vd", [(128, 128), (64, 128), (100, 80), (64, 64)])
@pytest.mark.parametrize("lengths", [[1100, 333, 128], [90, 17, 260]])
def test_norms_of_what_is_off(lengths, kd, vd, name):
    c = Case(lengths, 3, kd, vd, name, decays=DECAYS, scale=0.3 * kd ** -0.5, seed=11)
    c.run()
    c.check()
    ends = torch.tensor([0] + lengths).cumsum(0).tolist()
    for i, (value, _) in enumerate(c.reference()):
        for h in range(3):
            for x, summary in (("last", c.summary), ("dfirst", c.dsummary)):
                got = summary[i, 3:].double().view(3, kd, vd)[h]
                assert (got - value[x][h]).norm() <= 2.0 ** -20 * value[x][h].norm(), (x, i, h)
        for x in ("o", "dq", "dk", "dv"):
            got = c.inner(x)[ends[i]:ends[i + 1]].double().unflatten(1, (3, -1))
            own = (value[x].to(c.t).double() - value[x]).norm()
            limit = 2.0 ** -21 * value[x].norm() if name == "f32" else 1.5 * own
            assert (got - value[x]).norm() <= limit, (x, i)


def test_a_lost_part_would_be_seen():
    """The limit for states against sums whose numbers lack their last part: c times a weight in bf16's parts."""
    g = torch.Generator().manual_seed(1)
    w = torch.exp(torch.arange(128, 0, -1).double() * torch.log(torch.tensor(DECAYS[0]).double())) * 0.3
    c, b = (torch.randn(128, 64, generator=g).bfloat16().double() for _ in range(2))
    bf = lambda x: x.bfloat16().double()  # noqa: E731
    w1 = bf(w)
    w2 = bf(w - w1)
    w3 = bf(w - w1 - w2)
    assert ((w - w1 - w2 - w3).abs() <= 2.0 ** -26 * w).all()
    parts = [bf(c * w1[:, None])]
    parts.append(bf(c * w1[:, None] - parts[0]))
    parts.append(bf(c * w2[:, None]))
    parts.append(bf(c * w2[:, None] - parts[2] + c * w3[:, None]))
    want = (c * w[:, None]).T @ b
    far = lambda p: ((sum(p).T @ b - want).norm() / want.norm()).item()  # noqa: E731
    assert far(parts) <= 2.0 ** -24 and all(far(parts[:i] + parts[i + 1:]) > 2.0 ** -20 for i in range(4))
