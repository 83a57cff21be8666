"""Batches of matrices that lie side by side in the rows of one buffer, as the column blocks of a fused projection:
the same bits as the matrices by themselves, nothing written beside them, and the layouts that are refused.
"""
import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_ortho import TYPES, matrices, planned


def refused(code, call, *args, **kw):
    with pytest.raises(sp.SparbitError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_layouts():
    a = [(i + 1) << 40 for i in range(4)]
    plan = sp.OrthoPlan(3, 64, 96, sp.BF16)
    run = lambda **kw: plan.orthogonalize(a[0], a[1], **kw)  # noqa: E731
    side = dict(ld=300, stride=100, out_ld=300, out_stride=100)
    refused(sp.ERR_WORKSPACE, run, **side)                       # as it should lie
    refused(sp.ERR_WORKSPACE, run, ld=296, stride=100)           # the last block ends with the row
    refused(sp.ERR_ARG, run, ld=295, stride=100)
    refused(sp.ERR_ARG, run, ld=300, stride=95)                  # blocks that overlap
    refused(sp.ERR_ARG, run, ld=300, stride=0)
    refused(sp.ERR_ARG, run, out_ld=300, out_stride=301)
    # another operator's columns of the same rows are not touched
    refused(sp.ERR_WORKSPACE, plan.orthogonalize, a[0], a[0] + 2 * 300, ld=600, stride=100, out_ld=600, out_stride=100)
    refused(sp.ERR_ALIAS, plan.orthogonalize, a[0], a[0] + 2 * 295, ld=600, stride=100, out_ld=600, out_stride=100)
    refused(sp.ERR_ALIAS, plan.orthogonalize, a[0], a[0] + 2 * 400, ld=600, stride=100, out_ld=600, out_stride=100)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,gap,pad", [(60, 100, 0, 0), (150, 90, 3, 5), (128, 64, 0, 64), (300, 96, 8, 0)])
def test_side_by_side(rows, cols, gap, pad, dtype):
    t, count = TYPES[dtype][1], 3
    u = matrices(count, rows, cols, seed=2).to(t)
    plan = planned(count, rows, cols, dtype)
    want = torch.empty_like(u)
    plan.orthogonalize(u, want)
    stride = cols + gap
    ld = count * stride + pad
    src = torch.full((rows, ld), float("nan"), dtype=t, device="cuda")
    dst = torch.full((rows, ld), 7.0, dtype=t, device="cuda")
    view = lambda b: b.as_strided((count, rows, cols), (stride, ld, 1))  # noqa: E731
    view(src).copy_(u)
    plan.orthogonalize(src, dst, ld=ld, stride=stride, out_ld=ld, out_stride=stride)
    assert plan.status() == sp.OK
    assert torch.equal(view(dst), want)
    view(dst).fill_(7.0)
    assert (dst == 7.0).all()


@pytest.mark.gpu
def test_muon_step_of_column_blocks():
    count, rows, cols = 3, 96, 64
    g = matrices(count, rows, cols, seed=1).bfloat16()
    m, w = matrices(count, rows, cols, seed=2), matrices(count, rows, cols, seed=3, scale=0.02)
    plan = planned(count, rows, cols, "bf16")
    m2, w2 = torch.empty_like(m), torch.empty_like(w)
    kw = dict(weight_dtype=sp.F32, lr=0.1, weight_decay=0.1)
    plan.muon_step(g, m, m2, w, w2, **kw)
    fused = lambda v: v.permute(1, 0, 2).reshape(rows, count * cols).contiguous()  # noqa: E731
    fg, fm, fw = fused(g), fused(m), fused(w)
    ld = count * cols
    plan.muon_step(fg, fm, fm, fw, fw, grad_ld=ld, grad_stride=cols, momentum_ld=ld, momentum_stride=cols, weight_ld=ld,
                   weight_stride=cols, **kw)
    assert plan.status() == sp.OK
    assert torch.equal(fm, fused(m2)) and torch.equal(fw, fused(w2))
