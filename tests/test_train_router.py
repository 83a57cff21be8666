"""The router on the GPU against the formulas in 64 bits.

Tolerances.  p is an exponential of a difference whose rounding is 2^-24 of the logit's size L, then
a sum of E terms by a tree and a division: relative error at most (2 L + 16) 2^-24 =: r.  Sums over n
tokens add their rounding, 2^-24 a step along a warp's run and the joins behind it: n / 8 + 32 steps
relative to the sum (all terms have one sign).  A gradient is a sum of three products of such terms:
8 r times the sum of their magnitudes, then half a unit of its type.  A weight below 2^-126, the
smallest normal number of 32 bits, may be anything between 0 and that.
"""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"f32": (sp.F32, torch.float32, 2.0 ** -24), "bf16": (sp.BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (sp.F16, torch.float16, 2.0 ** -11)}
EPS = 2.0 ** -24
ALPHA, BETA = 0.3, 0.02


def dev(*shape, dtype=torch.float32, fill=None):
    t = torch.empty(*shape, dtype=dtype, device="cuda")
    return t if fill is None else t.fill_(fill)


def reference(l, mask, tokens, k, renormalize, dw, dloss=1.0):
    """Everything in 64 bits on the CPU; l as the kernel sees it."""
    T, E = l.shape
    l = l.double()
    usable = l > -float("inf")     # false for NaN too
    on = mask & usable.any(1)
    idx = torch.full((T, k), -1, dtype=torch.int32)
    wgt, lse = torch.zeros(T, k, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    p = torch.zeros(T, E, dtype=torch.float64)
    for t in range(T):
        if not on[t]:
            continue
        lse[t] = torch.logsumexp(l[t], 0)
        p[t] = torch.exp(l[t] - lse[t])
        order = sorted((e for e in range(E) if usable[t, e]), key=lambda e: (-l[t, e].item(), e))[:k]
        idx[t, :len(order)] = torch.tensor(order, dtype=torch.int32)
        wgt[t, :len(order)] = p[t, order]
        if renormalize:
            wgt[t] /= wgt[t].sum()
    counts, sums, at = [], [], 0
    for n in tokens:
        part = slice(at, at + n)
        at += n
        c = torch.zeros(E + 1, dtype=torch.int64)
        for e in idx[part].reshape(-1).tolist():
            if e >= 0:
                c[e] += 1
        c[E] = int(on[part].sum())
        counts.append(c)
        sums.append(torch.cat([p[part].sum(0), (lse[part] ** 2).sum()[None]]))
    counts, sums = torch.stack(counts), torch.stack(sums)
    N = max(1, int(counts[:, E].sum()))
    f = counts[:, :E].sum(0).double() / (N * k)
    loss = ALPHA * E / N * (sums[:, :E] @ f) + BETA / N * sums[:, E]
    inner = (p * f).sum(1, keepdim=True)
    balance = dloss * ALPHA * E / N * p
    zterm = dloss * 2 * BETA / N * lse[:, None] * p
    d = balance * (f - inner) + zterm
    size = balance * (f + inner) + zterm.abs()
    safe = idx.clamp_min(0).long()
    if dw is not None:
        dw = torch.where(idx >= 0, dw.double(), 0.0)
        s = (dw * wgt).sum(1, keepdim=True)
        sa = (dw.abs() * wgt).sum(1, keepdim=True)
        d = d.scatter_add(1, safe, wgt * ((dw - s) if renormalize else dw))
        size = size.scatter_add(1, safe, wgt * (dw.abs() + (sa if renormalize else 0)))
        if not renormalize:
            d, size = d - p * s, size + p * sa
    return dict(idx=idx, wgt=wgt, lse=lse, counts=counts, sums=sums, loss=loss, d=d, size=size, on=on)


def logits_of(T, E, dtype, seed, ties=False):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) * 1.5
    if ties:
        l = torch.round(l)
    return l.to(TYPES[dtype][1])


def run(l, tokens, k, renormalize, dtype, mask=None, ld=None, stream=None, dloss=None, dw=True, seed=3):
    code, t, unit = TYPES[dtype]
    T, E = l.shape
    R = len(tokens)
    plan = sp.RouterPlan(tokens, E, k, code, renormalize=renormalize)
    ws = dev(max(1, plan.workspace_bytes), dtype=torch.uint8, fill=0xCD)
    plan.set_workspace(ws, ws.numel())
    ld = ld or E
    buf = torch.full((T + 1, ld), float("nan"), dtype=t, device="cuda")
    buf[:T, :E] = l.cuda()
    out = torch.full((T + 1, ld), 7.0, dtype=t, device="cuda")
    m = None if mask is None else mask.to(torch.uint8).cuda()
    idx, wgt, lse = dev(T, k, dtype=torch.int32, fill=-7), dev(T, k, fill=-7), dev(T, fill=-7)
    counts, sums, loss = dev(R, E + 1, dtype=torch.int32, fill=-7), dev(R, E + 1, fill=-7), dev(R, fill=-7)
    dwt = torch.randn(T, k, generator=torch.Generator().manual_seed(seed)) * 0.1 if dw else None
    dl = None if dloss is None else dev(1, fill=dloss)
    gather, gathered = sp.Plan(R, (E + 1) * 4), dev(R, R, E + 1, dtype=torch.int32)
    dwd = dwt.cuda() if dw else None
    torch.cuda.synchronize()
    plan.forward(buf, idx, wgt, lse, counts, sums, mask=m, ld=ld, stream=stream)
    gather.allgather(counts, gathered, stream=stream)
    plan.balance(gathered, R, sums, loss, alpha=ALPHA, beta=BETA, stream=stream)
    plan.backward(buf, idx, wgt, lse, gathered, R, out, dweights=dwd, alpha=ALPHA, beta=BETA, dloss=dl, mask=m, ld=ld,
                  dlogits_ld=ld, stream=stream)
    torch.cuda.synchronize()
    assert (out[T] == 7.0).all() and (out[:, E:] == 7.0).all()
    return dict(idx=idx.cpu(), wgt=wgt.double().cpu(), lse=lse.double().cpu(), counts=counts.cpu().long(),
                sums=sums.double().cpu(), loss=loss.double().cpu(), d=out[:T, :E].double().cpu(), dw=dwt)


def check(l, tokens, k, renormalize, dtype, mask=None, **kw):
    got = run(l, tokens, k, renormalize, dtype, mask=mask, **kw)
    m = torch.ones(l.shape[0], dtype=torch.bool) if mask is None else mask
    dloss = kw.get("dloss")
    want = reference(l, m, tokens, k, renormalize, got["dw"], 1.0 if dloss is None else dloss)
    usable = l.double()[torch.isfinite(l.double()) & m[:, None]]
    L = usable.abs().max().item() if usable.numel() else 0.0
    r = (2 * L + 16) * EPS
    unit = TYPES[dtype][2]
    assert torch.equal(got["idx"], want["idx"])
    assert torch.equal(got["counts"], want["counts"])
    ok = lambda a, b, lim: ((a - b).abs() <= lim).all()  # noqa: E731
    assert ok(got["wgt"], want["wgt"], 3 * r * want["wgt"] + 2.0 ** -126)
    assert ok(got["lse"], want["lse"], (L + 8) * 4 * EPS)
    n = max(tokens)
    rs = r + (n / 8 + 32) * EPS
    assert ok(got["sums"], want["sums"], 4 * rs * want["sums"] + 1e-30)
    assert ok(got["loss"], want["loss"], 8 * rs * want["loss"] + 1e-30)
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-38
    assert ok(got["d"], want["d"], 8 * r * want["size"] + unit * want["d"].abs() + tiny)
    return got, want


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (8, 2), (31, 5), (32, 32), (33, 3), (60, 4), (64, 6), (65, 8), (128, 8),
                                 (129, 1), (256, 8), (300, 10), (512, 12), (513, 7), (1024, 32)])
def test_experts(E, k, dtype):
    check(logits_of(70, E, dtype, E), [70], k, E % 2 == 0, dtype)


@pytest.mark.parametrize("tokens", [[1], [0], [0, 3, 0], [7, 8, 9, 1], [640, 33], [5000]], ids=str)
@pytest.mark.parametrize("renormalize", [False, True])
def test_ranks_and_tokens(tokens, renormalize):
    check(logits_of(sum(tokens), 20, "bf16", 1), tokens, 3, renormalize, "bf16")


@pytest.mark.parametrize("dtype", list(TYPES))
def test_equal_logits_take_the_lowest_expert_first(dtype):
    check(logits_of(300, 64, dtype, 2, ties=True), [300], 6, False, dtype)
    check(torch.zeros(5, 64, dtype=TYPES[dtype][1]), [5], 6, True, dtype)
    l = torch.zeros(4, 40, dtype=TYPES[dtype][1])
    l[:, ::2] = -0.0     # minus zero and zero are equal
    check(l, [4], 5, True, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("renormalize", [False, True])
def test_left_out_tokens_reach_nothing(dtype, renormalize):
    l = logits_of(200, 48, dtype, 4)
    mask = torch.rand(200, generator=torch.Generator().manual_seed(0)) > 0.4
    l[~mask] = float("nan")
    l[5] = float("inf")
    mask[5] = False
    check(l, [120, 80], 4, renormalize, dtype, mask=mask)
    check(l, [120, 80], 4, renormalize, dtype, mask=torch.zeros(200, dtype=torch.bool))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("renormalize", [False, True])
def test_experts_that_are_masked(dtype, renormalize):
    """-inf in some places, in all but fewer than k, and in a whole row; the type's lowest value is a value."""
    l = logits_of(60, 40, dtype, 5)
    l[:20, 10:] = float("-inf")
    l[20:30, 2:] = float("-inf")
    l[30:33] = float("-inf")
    check(l, [25, 35], 6, renormalize, dtype)
    low = logits_of(10, 40, dtype, 6)
    low[:, 3:] = torch.finfo(low.dtype).min
    got = run(low, [10], 6, renormalize, dtype)
    assert (got["idx"] >= 0).all() and torch.isfinite(got["d"]).all() and torch.isfinite(got["wgt"]).all()
    assert torch.equal(got["idx"][:, 3:], torch.arange(3, 6, dtype=torch.int32).expand(10, 3))


def test_nan_in_a_token_that_takes_part():
    l = logits_of(20, 40, "f32", 5)
    l[7, 3] = float("nan")
    got = run(l, [20], 4, False, "f32")
    assert torch.isnan(got["wgt"][7]).all() and torch.isnan(got["lse"][7]) and torch.isnan(got["d"][7]).all()
    assert not (got["idx"][7] == 3).any() and (got["idx"][7] >= 0).all()
    others = [t for t in range(20) if t != 7]
    assert torch.isfinite(got["wgt"][others]).all() and torch.isfinite(got["lse"][others]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,ld", [(64, 72), (64, 65), (60, 64), (256, 264), (33, 40)])
def test_row_strides(E, ld, dtype):
    check(logits_of(90, E, dtype, 9), [90], 4, True, dtype, ld=ld)


def test_large_logits_and_scales():
    l = (logits_of(100, 64, "f32", 1) * 30).float()
    check(l, [100], 8, True, "f32", dloss=3.0)
    check(l, [100], 8, False, "f32", dw=False)


def test_a_stream_of_ones_own_and_again():
    l, stream = logits_of(3000, 128, "bf16", 8), torch.cuda.Stream()
    a, _ = check(l, [1000, 2000], 8, True, "bf16", stream=stream)
    b, _ = check(l, [1000, 2000], 8, True, "bf16", stream=stream)
    for key in ("sums", "loss", "d", "wgt"):
        assert torch.equal(a[key], b[key]), key


def test_gradient_against_differences():
    tokens, E, k = [30, 20], 24, 3
    l = logits_of(50, E, "f32", 11)
    for renormalize in (False, True):
        got = run(l, tokens, k, renormalize, "f32")
        base = reference(l, torch.ones(50, dtype=torch.bool), tokens, k, renormalize, got["dw"])
        N = 50
        f = base["counts"][:, :E].sum(0).double() / (N * k)
        safe = base["idx"].long()

        def value(x):
            p = torch.softmax(x, 1)
            w = p.gather(1, safe)
            if renormalize:
                w = w / w.sum(1, keepdim=True)
            return (ALPHA * E / N * (p.sum(0) * f).sum() + BETA / N * (torch.logsumexp(x, 1) ** 2).sum()
                    + (got["dw"].double() * w).sum()).item()

        gen = torch.Generator().manual_seed(2)
        for _ in range(4):
            way = torch.randn(l.shape, generator=gen, dtype=torch.float64)
            eps = 1e-4
            want = (value(l.double() + eps * way) - value(l.double() - eps * way)) / (2 * eps)
            terms = got["d"] * way
            assert abs(terms.sum().item() - want) <= 1e-5 * terms.abs().sum().item()


def test_counts_size_an_allgatherv():
    """The gathered counts are the block sizes of what the ranks exchange next."""
    tokens, E, k = [40, 13, 27], 16, 2
    got, _ = check(logits_of(80, E, "f32", 12), tokens, k, False, "f32")
    sent = got["counts"][:, :E].sum(1)
    assert sent.tolist() == [n * k for n in tokens]
    plan = sp.Plan.create_v([4 * int(n) for n in sent])
    blocks = dev(int(sent.sum()), dtype=torch.int32)
    blocks.copy_(got["idx"].reshape(-1))
    out = dev(3, int(sent.sum()), dtype=torch.int32)
    plan.allgather(blocks, out)
    assert plan.status() == sp.OK
    assert all(torch.equal(out[r], blocks) for r in range(3))
