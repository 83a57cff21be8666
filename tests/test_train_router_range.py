"""The router over the whole range of its types: logits of any magnitude are logits, the type's lowest value as
much as another.

Tolerances.  p depends on differences of logits, which the cases here hold exactly (equal logits, or small
multiples of a power of two apart), so that their size does not enter: with d the largest finite difference, d log2(e)
is rounded to 2^-24 of itself, then an exponential, a sum of E terms by a tree and a division follow: r =
(2 d + 16) 2^-24 at most.  Where the gradient takes p from lse, whose rounding is 2^-24 of its size, that size
is at most 128: r' = (2 (128 + d) + 16) 2^-24.  lse itself and its square are good to 4 and 8 units of 2^-24; squares
beyond 32 bits are infinite.  Sums and losses are sums of such terms of one sign: (n + 32) 2^-24 more.  A
gradient is a sum of three products: 8 r' times the sum of their magnitudes, then half a unit of its type.
"""
import pytest
import torch

import test_train_router as router
from test_train_router import EPS, TYPES, logits_of, run

pytestmark = pytest.mark.gpu

BIG = 3.4028234663852886e38   # the largest number of 32 bits
FAR = {"f32": [-3e4, 1e9, -1e9, 1e10, -1e10, 1e30, -1e30, BIG, -BIG], "f16": [3e4, -3e4, 65504.0, -65504.0]}
FAR["bf16"] = FAR["f32"][:-2] + [torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min]


def in_64_bits(l, mask, tokens, k, renormalize, dw, beta, dloss=1.0):
    """The formulas, p taken from differences to the largest logit."""
    T, E = l.shape
    l = l.double()
    on = mask & (l > -float("inf")).any(1)
    x = torch.where(on[:, None], l, 0.0)
    top = x.max(1, keepdim=True).values
    part = torch.exp(x - top)
    p = torch.where(on[:, None], part / part.sum(1, keepdim=True), 0.0)
    lse = torch.where(on, top[:, 0] + torch.log(part.sum(1)), 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    usable = on[:, None] & (x.gather(1, order) > -float("inf"))
    idx = torch.where(usable, order, -1)
    wgt = torch.where(usable, p.gather(1, order), 0.0)
    if renormalize:
        wgt = torch.where(on[:, None], wgt / wgt.sum(1, keepdim=True), 0.0)
    rank = torch.repeat_interleave(torch.arange(len(tokens)), torch.tensor(tokens))
    counts = torch.zeros(len(tokens), E + 1, dtype=torch.int64)
    sums = torch.zeros(len(tokens), E + 1, dtype=torch.float64)
    for t in range(T):
        for e in idx[t].tolist():
            if e >= 0:
                counts[rank[t], e] += 1
        counts[rank[t], E] += int(on[t])
        sums[rank[t], :E] += p[t]
        sums[rank[t], E] += lse[t] ** 2
    N = max(1, int(counts[:, E].sum()))
    f = counts[:, :E].sum(0).double() / (N * k)
    alpha = router.ALPHA
    inner = (p * f).sum(1, keepdim=True)
    balance, zterm = dloss * alpha * E / N * p, dloss * 2 * beta / N * lse[:, None] * p
    d, size = balance * (f - inner) + zterm, balance * (f + inner) + zterm.abs()
    dw = torch.where(idx >= 0, dw.double(), 0.0)
    s, sa = (dw * wgt).sum(1, keepdim=True), (dw.abs() * wgt).sum(1, keepdim=True)
    at = idx.clamp_min(0)
    d = d.scatter_add(1, at, wgt * ((dw - s) if renormalize else dw))
    size = size.scatter_add(1, at, wgt * (dw.abs() + (sa if renormalize else 0)))
    if not renormalize:
        d, size = d - p * s, size + p * sa
    return dict(idx=idx.int(), wgt=wgt, lse=lse, counts=counts, sums=sums,
                alone=alpha * E / N * (sums[:, :E] @ f), squares=beta / N * sums[:, E], d=d, size=size, on=on)


def check(l, tokens, k, renormalize, dtype, difference, mask=None, beta=None, monkeypatch=None, **kw):
    beta = router.BETA if beta is None else beta
    if monkeypatch:
        monkeypatch.setattr(router, "BETA", beta)
    got = run(l, tokens, k, renormalize, dtype, mask=mask, **kw)
    m = torch.ones(l.shape[0], dtype=torch.bool) if mask is None else mask
    want = in_64_bits(l, m, tokens, k, renormalize, got["dw"], beta)
    r, rb = (2 * difference + 16) * EPS, (2 * (128 + difference) + 16) * EPS
    assert torch.equal(got["idx"], want["idx"])
    assert torch.equal(got["counts"], want["counts"])
    ok = lambda a, b, lim: ((a - b).abs() <= lim).all()  # noqa: E731
    assert ok(got["wgt"], want["wgt"], 3 * r * want["wgt"] + 2.0 ** -126)
    assert ok(got["lse"], want["lse"], 4 * EPS * want["lse"].abs() + 16 * EPS)
    E, n = l.shape[1], max(tokens)
    rs = r + (n + 32) * EPS
    assert ok(got["sums"][:, :E], want["sums"][:, :E], 4 * rs * want["sums"][:, :E] + 1e-30)
    lost = want["sums"][:, E] > BIG
    assert (got["sums"][lost, E] == float("inf")).all()
    assert ok(got["sums"][~lost, E], want["sums"][~lost, E], (4 * rs + 16 * EPS) * want["sums"][~lost, E] + 1e-30)
    loss = want["alone"] + want["squares"]
    if beta == 0:
        lost = torch.zeros_like(lost)
    assert (got["loss"][lost] == float("inf")).all()
    assert ok(got["loss"][~lost], loss[~lost], (8 * rs + 16 * EPS) * loss[~lost] + 1e-30)
    unit = TYPES[dtype][2]
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-38
    assert ok(got["d"], want["d"], 8 * rb * want["size"] + unit * want["d"].abs() + tiny)
    return got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("E,k", [(8, 2), (20, 3), (128, 12), (257, 8), (500, 32)])
def test_rows_of_one_value(E, k, dtype, renormalize):
    """A token all of whose experts were masked by a large negative number: each expert gets 1/E."""
    t = TYPES[dtype][1]
    for value in FAR[dtype]:
        check(torch.full((11, E), value, dtype=t), [11], k, renormalize, dtype, 0)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,k", [(20, 3), (60, 9), (300, 8)])
def test_far_rows_among_ordinary_ones(E, k, dtype):
    """The tokens of a warp do not touch one another: ordinary ones keep their bits, far ones are right."""
    l = logits_of(90, E, dtype, E)
    mixed = l.clone()
    for i, value in enumerate(FAR[dtype] * 2):
        mixed[5 * i + i % 3] = value
    ordinary = (mixed == l).all(1)
    difference = 2 * l.double().abs().max().item()
    for mask in (None, torch.rand(90, generator=torch.Generator().manual_seed(1)) > 0.3):
        got = check(mixed, [50, 40], k, True, dtype, difference, mask=mask)
        alone = run(l, [50, 40], k, True, dtype, mask=mask)
        for key in ("idx", "wgt", "lse"):
            assert torch.equal(got[key][ordinary], alone[key][ordinary]), key


@pytest.mark.parametrize("base", [-2.0 ** 20, -2.0 ** 14, -1000.0, 150.0, 2.0 ** 13, 2.0 ** 17])
@pytest.mark.parametrize("renormalize", [False, True])
def test_differences_count_wherever_they_lie(base, renormalize):
    """Multiples of 1/8 on top of a large number, exact in 32 bits."""
    l = torch.randint(-40, 40, (64, 48), generator=torch.Generator().manual_seed(2)).float() / 8 + base
    check(l, [64], 6, renormalize, "f32", 10)
    l[:, 30:] = -1e30
    check(l, [64], 6, renormalize, "f32", 10)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_fewer_ordinary_logits_than_choices(dtype):
    """Places after the ordinary logits go to the lowest experts of the masked value, with weight 0."""
    l = logits_of(40, 24, dtype, 3)
    l[:, 2:] = torch.finfo(l.dtype).min
    got = check(l, [40], 5, False, dtype, 10 if dtype != "f16" else 20)
    assert torch.equal(got["idx"][:, 2:], torch.arange(2, 5, dtype=torch.int32).expand(40, 3))
    assert (got["wgt"][:, 2:] == 0).all()


def test_no_weight_on_the_squares_is_no_weight(monkeypatch):
    """beta = 0: squares of lse that 32 bits do not hold stay out of the loss."""
    l = logits_of(30, 16, "f32", 7)
    l[4] = -1e30
    check(l, [30], 2, True, "f32", 20, beta=0.0, monkeypatch=monkeypatch)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_an_infinite_logit_is_like_a_nan(dtype):
    """inf - inf: the token's weights, lse and gradient are NaN, it is chosen first, other tokens are as ever."""
    l = logits_of(20, 40, dtype, 5)
    plain = run(l, [20], 4, False, dtype)
    l[7, 3] = float("inf")
    got = run(l, [20], 4, False, dtype)
    assert torch.isnan(got["wgt"][7]).all() and torch.isnan(got["lse"][7]) and torch.isnan(got["d"][7]).all()
    assert got["idx"][7, 0] == 3
    others = [t for t in range(20) if t != 7]
    for key in ("idx", "wgt", "lse"):
        assert torch.equal(got[key][others], plain[key][others])
