"""The orthogonalised update on the GPU against the iteration in 64 bits.

Tolerances, in the Frobenius norm relative to the result.  In one step the operands P and X of the
last product are rounded to u (2^-11 for one product, 2^-21 for three), each of which moves the
result by at most |P| u |X|, |P| < 2.8 with the usual coefficients; near singular values of one a
step carries an error on with a factor of about one, so five steps make at most 5 * 2 * 2.8 u of the
result: 1.4e-2 for one product, 1.4e-5 for three.  fp32 accumulation over K terms adds about
sqrt(K) 2^-24 a product, 6e-6 for the largest K here and five steps of three products.  The result's
own rounding, u_type, comes on top.
"""
import math

import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"f32": (sp.F32, torch.float32, 2.0 ** -24), "bf16": (sp.BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (sp.F16, torch.float16, 2.0 ** -11)}
QUINTIC = (3.4445, -4.7750, 2.0315)
LIMIT = {1: 1.4e-2, 3: 2e-5}


def reference(u, steps=5, coefficients=None, eps=1e-7):
    u = u.double()
    x = u / (u.square().sum((-1, -2), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT
    for i in range(steps):
        a, b, c = coefficients[i] if coefficients else QUINTIC
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def matrices(count, rows, cols, kind="random", seed=0, scale=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if kind == "random":
        return r(count, rows, cols) * scale
    if kind == "decay":
        k = min(rows, cols)
        left = r(count, rows, k) / torch.arange(1, k + 1, device="cuda")
        return torch.bmm(left, r(count, k, cols)) * scale
    k = max(1, min(rows, cols) // 8)
    return torch.bmm(r(count, rows, k), r(count, k, cols)) * scale


def planned(count, rows, cols, dtype, products=None, **kw):
    plan = sp.OrthoPlan(count, rows, cols, TYPES[dtype][0], **kw)
    if products:
        plan.set_products(products)
    ws = torch.full((plan.workspace_bytes,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN wherever it is read as a float
    plan.set_workspace(ws, ws.numel())
    return plan


def far(got, want):
    """The worst relative distance of the matrices of a batch."""
    d = (got.double() - want).square().sum((-1, -2)).sqrt() / want.square().sum((-1, -2)).sqrt()
    return d.max().item()


def check(count, rows, cols, dtype, kind="random", products=None, seed=0, scale=1e-3, **kw):
    t, unit = TYPES[dtype][1:]
    u = matrices(count, rows, cols, kind, seed, scale).to(t)
    plan = planned(count, rows, cols, dtype, products, **kw)
    out = torch.full((count * rows * cols + 64,), 7.0, dtype=t, device="cuda")
    plan.orthogonalize(u, out)
    assert plan.status() == sp.OK
    assert (out[count * rows * cols:] == 7.0).all()
    got = out[:count * rows * cols].view(count, rows, cols)
    n = products or (1 if dtype == "bf16" else 3)
    want = reference(u, **{k: v for k, v in kw.items() if k in ("steps", "coefficients", "eps")})
    d = far(got, want)
    assert d <= LIMIT[n] + unit, d
    return d


SIZES = [(1, 1), (1, 7), (7, 1), (8, 8), (63, 65), (64, 64), (65, 200), (127, 129), (128, 128), (129, 128), (130, 257),
         (256, 256), (255, 513), (300, 1000), (1000, 300), (512, 640), (700, 701)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, dtype):
    check(1, rows, cols, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("count,rows,cols", [(3, 40, 72), (5, 130, 70), (2, 300, 260), (33, 64, 64)])
def test_batches(count, rows, cols, dtype):
    check(count, rows, cols, dtype, seed=4)


@pytest.mark.parametrize("dtype,products", [("bf16", 1), ("bf16", 3), ("f16", 3), ("f32", 1), ("f32", 3)])
@pytest.mark.parametrize("kind", ["random", "lowrank", "decay"])
def test_numbers_of_products(dtype, products, kind):
    check(1, 200, 500, dtype, kind=kind, products=products)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e20, 1e34])
def test_magnitudes(scale):
    """The norm is taken in 64 bits and divided out by a power of two first; eps counts only where it matters."""
    check(1, 100, 150, "f32", scale=scale, eps=0.0)
    check(1, 100, 150, "bf16", scale=scale, eps=0.0)
    if scale == 1e-12:
        check(1, 100, 150, "f32", scale=scale, eps=1e-10)


@pytest.mark.parametrize("steps,coefficients", [(1, [(1.875, -1.25, 0.375)]), (12, [(1.875, -1.25, 0.375)] * 12),
                                                (3, [(3.0, -3.2, 1.2), QUINTIC, (1.5, -0.5, 0.0)])])
def test_coefficients(steps, coefficients):
    check(1, 90, 140, "f32", steps=steps, coefficients=coefficients)
    check(1, 90, 140, "bf16", steps=steps, coefficients=coefficients)


def test_converges_to_the_orthogonal_factor():
    """With a convergent iteration X X^T becomes the identity."""
    plan = planned(1, 64, 200, "f32", steps=14, coefficients=[(1.875, -1.25, 0.375)] * 14)
    u, out = matrices(1, 64, 200)[0], torch.empty(64, 200, device="cuda")
    plan.orthogonalize(u, out)
    eye = torch.eye(64, dtype=torch.float64, device="cuda")
    assert (out.double() @ out.double().T - eye).norm().item() / 8 < 2e-5


def test_zero_and_not_finite():
    u = matrices(4, 70, 90).to(torch.bfloat16)
    u[1] = 0
    u[2, 3, 4] = float("nan")
    u[3, 69, 89] = float("inf")
    plan = planned(4, 70, 90, "bf16")
    out = torch.empty_like(u)
    plan.orthogonalize(u, out)
    assert far(out[:1], reference(u[:1])) <= LIMIT[1] + 2.0 ** -8
    assert (out[1] == 0).all()
    assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(60, 100), (150, 90)])
def test_strides(rows, cols, dtype):
    t, unit = TYPES[dtype][1:]
    u = matrices(3, rows, cols, seed=2).to(t)
    plan = planned(3, rows, cols, dtype)
    for pad, gap, shift in ((5, 0, 1), (8, 3, 0), (0, 17, 0)):
        ld = cols + pad
        stride = rows * ld + gap
        src = torch.full((3 * stride + shift,), float("nan"), dtype=t, device="cuda")
        dst = torch.full((3 * stride + shift,), 7.0, dtype=t, device="cuda")
        view = lambda b: b[shift:].as_strided((3, rows, cols), (stride, ld, 1), shift)  # noqa: E731
        view(src).copy_(u)
        plan.orthogonalize(src[shift:], dst[shift:], ld=ld, stride=stride, out_ld=ld, out_stride=stride)
        assert far(view(dst), reference(u)) <= LIMIT[1 if dtype == "bf16" else 3] + unit
        view(dst).fill_(7.0)
        assert (dst == 7.0).all()


@pytest.mark.parametrize("dtype,weights", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols", [(96, 160), (300, 130)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon(rows, cols, dtype, weights, nesterov):
    t, wt, unit = TYPES[dtype][1], TYPES[weights][1], TYPES[weights][2]
    g = matrices(2, rows, cols, seed=1).to(t)
    m, w = matrices(2, rows, cols, seed=2, scale=5e-4), (matrices(2, rows, cols, seed=3, scale=0.02)).to(wt)
    plan = planned(2, rows, cols, dtype)
    lr, mu, decay, scale = 0.03, 0.9, 0.1, 0.2 * math.sqrt(max(rows, cols))
    want_m = mu * m.double() + g.double()
    x = reference(g.double() + mu * want_m if nesterov else want_m)
    want_w = (1 - lr * decay) * w.double() - lr * scale * x
    m2, w2 = torch.empty_like(m), torch.empty_like(w)
    kw = dict(weight_dtype=TYPES[weights][0], lr=lr, momentum=mu, nesterov=nesterov, weight_decay=decay, scale=scale)
    plan.muon_step(g, m, m2, w, w2, **kw)
    assert ((m2.double() - want_m).abs() <= 4 * 2.0 ** -24 * (m.double().abs() + g.double().abs())).all()
    step = lr * scale * x.square().sum().sqrt().item()
    lim = (LIMIT[1 if dtype == "bf16" else 3]) * step + (unit + 4 * 2.0 ** -24) * want_w.norm().item()
    assert (w2.double() - want_w).norm().item() <= lim
    # in place, the same bits
    plan.muon_step(g, m, m, w, w, **kw)
    assert torch.equal(m, m2) and torch.equal(w, w2)


def test_a_stream_of_ones_own_again_and_in_a_graph():
    plan = planned(2, 200, 333, "bf16")
    u = matrices(2, 200, 333).to(torch.bfloat16)
    first, second = torch.empty_like(u), torch.empty_like(u)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan.orthogonalize(u, first, stream=stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        plan.orthogonalize(u, second, stream=stream)
    for _ in range(5):
        second.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, second)


def test_rows_gathered_by_the_library_itself():
    """A receive buffer of the allgather is the matrix: every rank orthogonalises the same one."""
    P, each, cols = 4, 24, 130
    u = matrices(1, P * each, cols)[0].to(torch.bfloat16)
    gather = sp.Plan(P, each * cols * 2)
    recv = torch.empty(P, P * each, cols, dtype=torch.bfloat16, device="cuda")
    gather.allgather(u, recv)
    plan = planned(P, P * each, cols, "bf16")
    out = torch.empty_like(recv)
    plan.orthogonalize(recv, out)
    assert gather.status() == sp.OK and plan.status() == sp.OK
    assert far(out, reference(u[None])) <= LIMIT[1] + 2.0 ** -8
    assert all(torch.equal(out[r], out[0]) for r in range(P))
