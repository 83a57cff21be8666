"""Addresses that are no multiples of their elements' sizes, which a kernel could not read, are refused on the host, no GPU."""
import pytest

import paper_2109_08751_b200 as sp
from test_train_host import GPU_SIZED, refused

A = [GPU_SIZED * (i + 1) for i in range(16)]


def odd(call, given, sizes):
    """Every argument by itself half an element further on."""
    for name, size in sizes.items():
        refused(sp.ERR_ARG, call, **{**given, name: given[name] + size // 2})


@pytest.mark.parametrize("code,size", [(sp.F32, 4), (sp.BF16, 2), (sp.F16, 2)])
def test_linear_attention(code, size):
    plan = sp.LinearAttentionPlan([100, 28], 2, 64, 32, code)
    names = dict(q=size, k=size, v=size, log_decay=4, o=size, first=4, summary=4)
    given = dict(zip(names, A))
    refused(sp.ERR_WORKSPACE, plan.forward, **given)
    odd(plan.forward, given, names)
    names = dict(q=size, k=size, v=size, log_decay=4, do=size, dq=size, dk=size, dv=size, first=4, dlast=4, dsummary=4)
    given = dict(zip(names, A))
    refused(sp.ERR_WORKSPACE, plan.backward, **given)
    odd(plan.backward, given, names)
    # what is not read may lie anywhere
    refused(sp.ERR_WORKSPACE, plan.forward, q=A[0] + 1, k=A[1], v=A[2], log_decay=A[3], o=None, summary=A[4])
    names = dict(q=size, k=size, v=size, log_decay=4, state_in=4, state_out=4, o=size, slots=4)
    odd(lambda **kw: sp.linear_attention_step(3, 2, 64, 32, code, n_slots=3, **kw), dict(zip(names, A)), names)
    names = dict(gathered=4, out=4, first=4)
    odd(lambda **kw: sp.linear_attention_join(4, 2, 64, 32, **kw), dict(zip(names, A)), names)


@pytest.mark.parametrize("code,size", [(sp.F32, 4), (sp.BF16, 2), (sp.F16, 2)])
def test_norm(code, size):
    for weight, of in ((code, size), (sp.F32, 4)):
        plan = sp.NormPlan(64, code, weight_dtype=weight)
        names = dict(x=size, weight=of, residual=size, sum=size, y=size, scales=4, rstd=4)
        odd(lambda **kw: plan.forward(10, y8=A[9] + 1, **kw), dict(zip(names, A)), names)
        names = dict(dy=size, sum=size, weight=of, rstd=4, dx=size, dweight=4, dsum=size)
        given = dict(zip(names, A))
        refused(sp.ERR_WORKSPACE, plan.backward, 10, **given)
        odd(lambda **kw: plan.backward(10, **kw), given, names)


def test_clip():
    plan = sp.ClipPlan([100], [sp.F32])
    refused(sp.ERR_ARG, plan.sums, A[0] + 4)
    refused(sp.ERR_ARG, plan.scale, A[0] + 4, 1, 1.0, A[1])
    refused(sp.ERR_ARG, plan.scale, A[0], 1, 1.0, A[1] + 2)
    refused(sp.ERR_WORKSPACE, plan.scale, A[0], 1, 1.0, A[1] + 4)
