"""The orthogonalised update at sizes whose products are many tiles: the 256-wide tiles, CTA pairs that take one tile
after another, and matrices near the error that is documented.

Which tiles a product takes is the library's rule, written down once more here, so that the cases are known to reach
them: the narrow ones (128) for three products and where rounds of 74 pairs of 1.3 times their width are fewer.

Tolerances, in the Frobenius norm relative to the result.  Operands are rounded to u = 2^-11 for one product and to
2^-21 for three, their errors independent of one another: u / sqrt(3) of their size.  The two operands of a step's last
product move the result by sqrt(2) 2.8 u / sqrt(3), five steps by sqrt(5) times that: 2.5e-3 for one product, of
which 3e-3 are allowed, and 2.4e-6 for three, to which partial sums in 32 bits add up to 2.5e-6: 5e-6 are allowed.
The result's own rounding, half a unit on average, comes on top.  (A linear term from hi alone would be 1e-2 off, partial sums left in the
tensor cores throughout 1e-5.)
"""
import math

import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_ortho import TYPES, far, matrices, planned, reference

pytestmark = pytest.mark.gpu

LIMIT = {1: 3e-3, 3: 5e-6}
PAIRS = 74


def tiles(rows, cols, width, square):
    down, across = -(-rows // 256), -(-cols // width)
    return sum(across - i * 256 // width for i in range(down)) if square else down * across


def layout(count, rows, cols, dtype):
    """(width, tiles of all matrices) of the symmetric products and of X."""
    m, n = min(rows, cols), max(rows, cols)
    out = []
    for c, square in ((m, True), (n, False)):
        wide, narrow = tiles(m, c, 256, square) * count, tiles(m, c, 128, square) * count
        is_narrow = dtype != "bf16" or -(-narrow // PAIRS) * 128 * 1.3 < -(-wide // PAIRS) * 256
        out.append((128, narrow) if is_narrow else (256, wide))
    return out


#: count, rows, cols, type, layout
CASES = [
    (1, 1024, 4096, "bf16", [(128, 20), (256, 64)]),
    (1, 1100, 4100, "bf16", [(128, 25), (128, 165)]),
    (1, 4100, 1100, "bf16", [(128, 25), (128, 165)]),
    (20, 700, 701, "bf16", [(256, 120), (256, 180)]),
    (20, 701, 700, "bf16", [(256, 120), (256, 180)]),
    (1, 2300, 2304, "bf16", [(256, 45), (128, 162)]),
    (20, 700, 701, "f32", [(128, 240), (128, 360)]),
    (3, 2100, 600, "f16", [(128, 27), (128, 153)]),
    (1, 512, 4096, "f32", [(128, 6), (128, 64)]),
]


@pytest.mark.parametrize("kind", ["random", "lowrank", "decay"])
@pytest.mark.parametrize("count,rows,cols,dtype,want", CASES, ids=str)
def test_many_tiles(count, rows, cols, dtype, want, kind):
    assert layout(count, rows, cols, dtype) == want
    t, unit = TYPES[dtype][1:]
    u = matrices(count, rows, cols, kind, seed=rows).to(t)
    plan = planned(count, rows, cols, dtype)
    out, again = torch.full_like(u, 7), torch.full_like(u, 7)
    plan.orthogonalize(u, out)
    plan.orthogonalize(u, again)
    assert plan.status() == sp.OK
    assert torch.equal(out, again)
    d = far(out, reference(u))
    assert d <= LIMIT[1 if dtype == "bf16" else 3] + unit / 2, d


@pytest.mark.parametrize("weights", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols,dtype,want", [c for c in CASES if c[0] == 20 or c[1] == 1024], ids=str)
def test_muon_step_of_many_tiles(count, rows, cols, dtype, want, weights):
    assert layout(count, rows, cols, dtype) == want
    t, wt, unit = TYPES[dtype][1], TYPES[weights][1], TYPES[weights][2]
    g = matrices(count, rows, cols, "lowrank", seed=1).to(t)
    m, w = matrices(count, rows, cols, seed=2, scale=5e-4), matrices(count, rows, cols, seed=3, scale=0.02).to(wt)
    lr, mu, decay, scale = 0.03, 0.9, 0.1, 0.2 * math.sqrt(max(rows, cols))
    want_m = mu * m.double() + g.double()
    x = reference(g.double() + mu * want_m)
    want_w = (1 - lr * decay) * w.double() - lr * scale * x
    plan = planned(count, rows, cols, dtype)
    plan.muon_step(g, m, m, w, w, weight_dtype=TYPES[weights][0], lr=lr, momentum=mu, weight_decay=decay, scale=scale)
    assert plan.status() == sp.OK
    assert ((m.double() - want_m).abs() <= 4 * 2.0 ** -24 * (want_m.abs() + g.double().abs())).all()
    each = lambda v: v.square().sum((-1, -2)).sqrt()  # noqa: E731
    lim = LIMIT[1 if dtype == "bf16" else 3] * lr * scale * each(x) + (unit / 2 + 2 * 2.0 ** -24) * each(want_w)
    assert (each(w.double() - want_w) <= lim).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(60, 20000), (200, 8000), (1024, 4096), (900, 900)])
def test_three_products_into_32_bit_weights(rows, cols, dtype):
    """The update that reaches 32-bit weights has the error of three products, whatever the gradient's type: sums
    are taken out of the tensor cores every block or two, which leaves 64 to 128 terms' worth of what they cut off, 3e-7
    of a product: 3e-6 with the operands' 2.4e-6."""
    t = TYPES[dtype][1]
    g = matrices(1, rows, cols, "decay", seed=1).to(t)
    plan = planned(1, rows, cols, dtype, products=3)
    m, w = torch.zeros(1, rows, cols, device="cuda"), torch.zeros(1, rows, cols, device="cuda")
    plan.muon_step(g, m, m, w, w, weight_dtype=sp.F32, lr=1.0, momentum=0.0, nesterov=False)
    assert plan.status() == sp.OK
    d = far(-w, reference(g))
    assert d <= 3e-6 + 2.0 ** -24, d
