"""Row strides and sizes that no matrix can have are refused on the host, no GPU: a negative stride arrives as a number
near 2^64, and offsets computed from it would wrap round to memory in front of the matrix.  (The addresses here are
numbers that nothing reads.)"""
import pytest

import paper_2109_08751_b200 as sp

A = [1 << 40 | i << 36 for i in range(12)]
WRONG = [-1, -16, -64, 1 << 46, 1 << 62, (1 << 63) + 64]


def refused(code, call, *args, **kw):
    with pytest.raises(sp.SparbitError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("ld", WRONG)
def test_scan(ld):
    plan = sp.ScanPlan([100, 28], 16, sp.BF16)
    forward = lambda **kw: plan.forward(A[0], A[1], A[2], h0=A[3], **kw)  # noqa: E731
    backward = lambda **kw: plan.backward(A[0], A[1], A[2], A[3], A[4], A[5], dlast=A[6], **kw)  # noqa: E731
    for name in ("gate_ld", "x_ld", "y_ld", "h0_ld"):
        refused(sp.ERR_ARG, forward, **{name: ld})
    for name in ("gate_ld", "x_ld", "dy_ld", "dgate_ld", "dx_ld", "dlast_ld"):
        refused(sp.ERR_ARG, backward, **{name: ld})
    refused(sp.ERR_WORKSPACE, forward, gate_ld=1 << 20, y_ld=1 << 20)   # far apart, and fine


@pytest.mark.parametrize("ld", WRONG)
def test_single_tokens_and_join(ld):
    step = lambda **kw: sp.scan_step(**{**dict(rows=4, channels=8, dtype=sp.F32, gate=A[0], x=A[1], state_in=A[2],  # noqa: E731
                                               state_out=A[2], y=A[3], slots=A[4], n_slots=9), **kw})
    for name in ("gate_ld", "x_ld", "y_ld", "state_ld"):
        refused(sp.ERR_ARG, step, **{name: ld})
    refused(sp.ERR_ARG, step, n_slots=-1)
    refused(sp.ERR_ARG, sp.scan_join, 4, 8, A[0], A[1], out_ld=ld)
    refused(sp.ERR_OVERFLOW, sp.scan_join, (1 << 31) - 1, 1 << 20, A[0], A[1], n_ranks=65535)


@pytest.mark.parametrize("ld", WRONG)
def test_router(ld):
    plan = sp.RouterPlan([100, 0, 5], 60, 4, sp.BF16)
    refused(sp.ERR_ARG, plan.forward, A[0], A[1], A[2], A[3], A[4], A[5], ld=ld)
    for name in ("ld", "dlogits_ld"):
        refused(sp.ERR_ARG, plan.backward, A[0], A[1], A[2], A[3], A[4], 3, A[5], **{name: ld})


@pytest.mark.parametrize("ld", WRONG)
def test_ortho(ld):
    plan = sp.OrthoPlan(2, 64, 96, sp.BF16)
    for name in ("ld", "out_ld", "stride", "out_stride"):
        refused(sp.ERR_ARG, plan.orthogonalize, A[0], A[1], **{name: ld})
    for name in ("grad_ld", "grad_stride", "momentum_ld", "momentum_stride", "weight_ld", "weight_stride"):
        refused(sp.ERR_ARG, plan.muon_step, A[0], A[1], A[1], A[2], A[2], weight_dtype=sp.F32, lr=0.1, **{name: ld})
