"""Root-mean-square norm with the residual's addition, its 8-bit rows and its gradients, against 64 bits.

Tolerances.  u: half a step of the type.  r is the rounded sum, to the bit.  y is 32-bit arithmetic (a sum of squares of at
most 2^15 numbers in a tree of partial sums of 32, a root, two factors: below 2^-19 of y) rounded once.  8-bit numbers:
half a step of e4m3 (2^-4 of the value, 2^-10 below its smallest normal number) of y over the scale, and what y and the
scale are off."""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, sp.BF16, 2.0 ** -8), "f16": (torch.float16, sp.F16, 2.0 ** -11),
         "f32": (torch.float32, sp.F32, 2.0 ** -24)}
EPS = 1e-6


def planned(width, name, **kw):
    plan = sp.NormPlan(width, TYPES[name][1], eps=EPS, **kw)
    work = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.set_workspace(work, work.numel())
    return plan


def rows_of(rows, width, t, g, pad=0, shift=0, std=1.0):
    wide = (torch.randn(rows, width + pad + shift, generator=g, device="cuda") * std).to(t)
    return wide[:, shift:shift + width]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width,pad,shift", [
    (1, 1, 0, 0), (3, 7, 0, 0), (5, 32, 0, 0), (130, 100, 0, 0), (9, 129, 3, 1), (1, 1000, 0, 0), (700, 1000, 0, 0),
    (2, 4096, 0, 0), (650, 4096, 8, 0), (650, 5000, 0, 0), (601, 5001, 2, 1), (3, 9000, 0, 0), (593, 9000, 0, 0),
    (2, 20000, 0, 0), (600, 16384, 0, 0), (2, 32768, 0, 0), (2000, 250, 0, 2)])
def test_forward_and_backward(rows, width, pad, shift, name):
    t, code, u = TYPES[name]
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    x, residual = rows_of(rows, width, t, g, pad, shift), rows_of(rows, width, t, g, pad, shift, 2.0)
    weight = (1 + 0.1 * torch.randn(width, generator=g, device="cuda")).to(t)
    at = dict(x_ld=width + pad + shift, residual_ld=width + pad + shift, sum_ld=width + 3, y_ld=width + 3)
    total, y = (torch.full((rows, width + 3), 7.0, dtype=t, device="cuda") for _ in range(2))
    rstd = torch.empty(rows, device="cuda")
    plan = planned(width, name)
    plan.forward(rows, x, weight, residual=residual, sum=total, y=y, rstd=rstd, **at)
    r = (x.float() + residual.float()).to(t)
    assert torch.equal(total[:, :width], r) and (total[:, width:] == 7.0).all() and (y[:, width:] == 7.0).all()
    k, w = r.double(), weight.double()
    s = 1 / (k.square().mean(1, keepdim=True) + EPS).sqrt()
    assert ((rstd.double()[:, None] - s).abs() <= 2.0 ** -20 * s).all()
    want = k * s * w
    assert ((y[:, :width].double() - want).abs() <= (u + 2.0 ** -19) * want.abs() + (2.0 ** -25 if name == "f16" else 0)).all()

    dy, dsum = rows_of(rows, width, t, g, pad, shift, 0.1), rows_of(rows, width, t, g, pad, shift, 0.1)
    dx, dweight = torch.full((rows, width + 3), 7.0, dtype=t, device="cuda"), torch.empty(width, device="cuda")
    plan.backward(rows, dy, total, weight, rstd, dx, dweight, dsum=dsum, dy_ld=dy.stride(0) if rows > 1 else width + pad + shift,
                  dsum_ld=width + pad + shift, sum_ld=width + 3, dx_ld=width + 3)
    d, n = dy.double() * w, k * s
    inner = (d * n).mean(1, keepdim=True)
    want = s * (d - n * inner) + dsum.double()
    size = s * (d.abs() + n.abs() * (d * n).abs().mean(1, keepdim=True)) + dsum.double().abs()
    assert ((dx[:, :width].double() - want).abs() <= u * want.abs() + 2.0 ** -18 * size + (2.0 ** -25 if name == "f16" else 0)).all()
    assert (dx[:, width:] == 7.0).all()
    want, size = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    assert ((dweight.double() - want).abs() <= 2.0 ** -18 * size).all()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width,block", [(1, 1, 0), (48, 4096, 128), (5, 100, 32), (700, 333, 64), (3, 5000, 0), (600, 5000, 256),
                                              (64, 64, 256), (9, 32, 32), (601, 9000, 0), (2, 20000, 128)])
def test_8_bit_rows(rows, width, block, name):
    t, code, u = TYPES[name]
    g = torch.Generator(device="cuda").manual_seed(rows * width)
    x = rows_of(rows, width, t, g)
    x[0, :] = 0  # a row of zeros
    if rows > 2:
        x[1, : width // 2] *= 1e-3
    weight = torch.randn(width, generator=g, device="cuda")
    plan = planned(width, name, weight_dtype=sp.F32, block=block)
    per_row = -(-width // block) if block else 1
    y8 = torch.full((rows, width + 5), 0x77, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.empty(rows, per_row, device="cuda")
    plan.forward(rows, x, weight, y8=y8, scales=scales, y8_ld=width + 5)
    k = x.double()
    y = k / (k.square().mean(1, keepdim=True) + EPS).sqrt() * weight.double()
    each = block or width
    amax = torch.stack([p.abs().amax(1) for p in y.split(each, 1)], 1)
    assert ((scales.double() - amax.clamp_min(1e-30) / 448).abs() <= 2.0 ** -18 * scales.double()).all()
    s = scales.double().repeat_interleave(each, 1)[:, :width]
    got = y8[:, :width].double()
    q = y / s
    assert ((got - q).abs() <= (2.0 ** -4 * q.abs()).clamp_min(2.0 ** -10) * (1 + 2.0 ** -10) + 2.0 ** -17 * q.abs()).all()
    assert (y8.view(torch.uint8)[:, width:] == 0x77).all()
    # the same rows with everything else written too
    both, yy, y8b, sb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(y8), torch.empty_like(scales)
    plan.forward(rows, x, weight, residual=torch.zeros_like(x), sum=both, y=yy, y8=y8b, scales=sb, y8_ld=width + 5)
    assert torch.equal(both, x) and torch.equal(sb, scales)
    assert torch.equal(y8b.view(torch.uint8)[:, :width], y8.view(torch.uint8)[:, :width])


def test_rows_that_32_bits_do_not_square():
    g = torch.Generator(device="cuda").manual_seed(0)
    for name, big in (("f32", 1e30), ("bf16", 1e30), ("f32", 3e38)):
        for width in (64, 4096):
            t = TYPES[name][0]
            x = rows_of(40, width, t, g)
            x[3] = (torch.randn(width, generator=g, device="cuda").clamp(-1, 1) * big).to(t)
            x[7] = float("nan")
            x[9, 5] = float("inf")
            x[11] *= 1e-20
            y = torch.empty_like(x)
            planned(width, name).forward(40, x, None, y=y)
            k = x.double()
            want = k / (k.square().mean(1, keepdim=True) + EPS).sqrt()
            fine = [i for i in range(40) if i not in (7, 9)]
            assert ((y[fine].double() - want[fine]).abs() <= (TYPES[name][2] + 2.0 ** -18) * want[fine].abs()).all()
            assert y[7].isnan().all() and y[9, 5].isnan() and (y[9, [i for i in range(width) if i != 5]] == 0).all()


def test_not_a_number_in_8_bits():
    x = torch.randn(4, 256, device="cuda")
    x[1, 40] = float("nan")
    plan = planned(256, "f32", block=64)
    y8, scales = torch.empty(4, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(4, 4, device="cuda")
    plan.forward(4, x, None, y8=y8, scales=scales)
    assert y8[1].float().isnan().all() and not scales[1].isfinite().any()
    assert y8[[0, 2, 3]].float().isfinite().all() and scales[[0, 2, 3]].isfinite().all()


@pytest.mark.parametrize("width", [96, 4096])
def test_in_place_and_on_a_stream_of_its_own(width):
    g = torch.Generator(device="cuda").manual_seed(4)
    x, r, dy, ds = (rows_of(900, width, torch.bfloat16, g) for _ in range(4))
    w, plan = torch.ones(width, dtype=torch.bfloat16, device="cuda"), planned(width, "bf16")
    outs = [torch.empty_like(x) for _ in range(3)]
    rstd, dw = torch.empty(900, device="cuda"), torch.empty(width, device="cuda")
    plan.forward(900, x, w, residual=r, sum=outs[0], y=outs[1], rstd=rstd)
    plan.backward(900, dy, outs[0], w, rstd, outs[2], dw, dsum=ds)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs] + [dw.clone()]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    x2, d2 = x.clone(), dy.clone()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        plan.forward(900, x2, w, residual=r, sum=x2, y=outs[1], rstd=rstd, stream=stream)
        plan.backward(900, d2, x2, w, rstd, d2, dw, dsum=ds, stream=stream)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x2, want[0]) and torch.equal(outs[1], want[1]) and torch.equal(d2, want[2]) and torch.equal(dw, want[3])
    # into the residual, and the gradient into dsum
    r2, s2 = r.clone(), ds.clone()
    plan.forward(900, x, w, residual=r2, sum=r2, rstd=rstd)
    plan.backward(900, dy, r2, w, rstd, s2, dsum=s2)
    assert torch.equal(r2, want[0]) and torch.equal(s2, want[2])


def test_gradient_against_differences():
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = rows_of(20, 50, torch.float32, g), rows_of(20, 50, torch.float32, g)
    w, plan = 1 + 0.1 * torch.randn(50, generator=g, device="cuda"), planned(50, "f32")
    y, rstd, dx, dw = torch.empty_like(x), torch.empty(20, device="cuda"), torch.empty_like(x), torch.empty(50, device="cuda")

    def loss(x, w):
        plan.forward(20, x, w, y=y, rstd=rstd)
        return (y.double() * dy.double()).sum()

    loss(x, w)
    plan.backward(20, dy, x, w, rstd, dx, dw)
    for t, grad, call in ((x, dx, lambda v: loss(v, w)), (w, dw, lambda v: loss(x, v))):
        way = torch.randn(t.shape, generator=g, device="cuda")
        h = 1e-2
        slope = ((call(t + h * way) - call(t - h * way)) / (2 * h)).item()
        want, size = (grad.double() * way.double()).sum().item(), (grad.double() * way.double()).abs().sum().item()
        assert abs(slope - want) <= 1e-3 * size  # h^2 of the third derivatives


def test_nothing_to_do():
    plan = planned(64, "bf16")
    dw = torch.full((64,), 7.0, device="cuda")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    plan.forward(0, e, None, y=e)
    plan.backward(0, e, e, None, torch.empty(0, device="cuda"), e, dw)
    assert (dw == 0).all()
