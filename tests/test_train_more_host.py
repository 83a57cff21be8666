"""Host side of linear attention, the norm and the clipping, no GPU: plans are made and refused as documented, argument
errors are found before anything is launched (the addresses here are numbers that nothing reads), and the binding makes
sure of types and gaps."""
import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_binding import OnTheGpu
from test_train_host import GPU_SIZED, refused

A = [GPU_SIZED * (i + 1) for i in range(16)]


def test_linear_attention_refusals():
    make = sp.LinearAttentionPlan
    refused(sp.ERR_ARG, make, [], 2, 64, 64)
    refused(sp.ERR_ARG, make, [4], 0, 64, 64)
    refused(sp.ERR_ARG, make, [4], 2, 0, 64)
    refused(sp.ERR_ARG, make, [4], 2, 64, 0)
    refused(sp.ERR_ARG, make, [4], 2, 64, 64, 5)
    refused(sp.ERR_ARG, make, [4], 2, 64, 64, scale=float("inf"))
    refused(sp.ERR_ARG, make, [4], 2, 64, 64, scale=float("nan"))
    refused(sp.ERR_LIMIT, make, [4], 2, 129, 64)
    refused(sp.ERR_LIMIT, make, [4], 2, 64, sp.LINEAR_ATTENTION_MAX_SIZE + 1)
    refused(sp.ERR_LIMIT, make, [4], 4097, 64, 64)
    refused(sp.ERR_LIMIT, make, [1 << 31], 1, 64, 64)
    refused(sp.ERR_OVERFLOW, make, [1 << 41], 1, 64, 64)
    with pytest.raises(ValueError):
        make([-1], 2, 64, 64)
    plan = make([100, 28], 2, 64, 32, sp.BF16)
    refused(sp.ERR_WORKSPACE, plan.set_workspace, A[0], 16)
    refused(sp.ERR_WORKSPACE, plan.set_workspace, A[0] + 8, 1 << 30)
    refused(sp.ERR_WORKSPACE, plan.status)
    forward = lambda **kw: plan.forward(**{**dict(q=A[0], k=A[1], v=A[2], log_decay=A[3], o=A[4], first=A[5],  # noqa: E731
                                                  summary=A[6]), **kw})
    refused(sp.ERR_WORKSPACE, forward)
    refused(sp.ERR_WORKSPACE, forward, q=None, o=None)
    refused(sp.ERR_WORKSPACE, forward, q=A[0], k=A[0] + 256, v=A[0] + 512, q_ld=320, k_ld=320, v_ld=320)
    refused(sp.ERR_ARG, forward, q=None)
    refused(sp.ERR_ARG, forward, k=None)
    refused(sp.ERR_ARG, forward, log_decay=None)
    refused(sp.ERR_ARG, forward, q_ld=127)
    refused(sp.ERR_ARG, forward, v_ld=63)
    refused(sp.ERR_ARG, forward, o_ld=1 << 62)
    refused(sp.ERR_ALIAS, forward, o=A[0])
    refused(sp.ERR_ALIAS, forward, summary=A[5] + 4)
    refused(sp.ERR_ALIAS, forward, summary=A[4] + 128 * 64 * 2 - 2)
    backward = lambda **kw: plan.backward(**{**dict(q=A[0], k=A[1], v=A[2], log_decay=A[3], do=A[4], dq=A[5], dk=A[6],  # noqa: E731
                                                    dv=A[7], first=A[8], dlast=A[9], dsummary=A[10]), **kw})
    refused(sp.ERR_WORKSPACE, backward)
    refused(sp.ERR_WORKSPACE, backward, dq=None, dk=None, dv=None, k=None, v=None)
    refused(sp.ERR_ARG, backward, dq=None)
    refused(sp.ERR_ARG, backward, dv=None)
    refused(sp.ERR_ARG, backward, do=None)
    refused(sp.ERR_ARG, backward, k=None)
    refused(sp.ERR_ARG, backward, dk_ld=1)
    refused(sp.ERR_ALIAS, backward, dq=A[4])
    refused(sp.ERR_ALIAS, backward, dk=A[5])
    refused(sp.ERR_ALIAS, backward, dsummary=A[9])
    step = lambda **kw: sp.linear_attention_step(**{**dict(rows=3, heads=2, key_size=64, value_size=32, dtype=sp.BF16, q=A[0],  # noqa: E731
                                                           k=A[1], v=A[2], log_decay=A[3], state_in=A[4], state_out=A[4],
                                                           o=A[5]), **kw})
    refused(sp.ERR_ARG, step, heads=0)
    refused(sp.ERR_ARG, step, dtype=7)
    refused(sp.ERR_ARG, step, q=None)
    refused(sp.ERR_ARG, step, state_out=None)
    refused(sp.ERR_ARG, step, n_slots=2)
    refused(sp.ERR_ARG, step, k_ld=100)
    refused(sp.ERR_ARG, step, scale=float("nan"))
    refused(sp.ERR_LIMIT, step, key_size=200)
    refused(sp.ERR_ALIAS, step, state_out=A[4] + 4)
    refused(sp.ERR_ALIAS, step, o=A[4])
    refused(sp.ERR_ALIAS, step, state_in=A[5], state_out=A[0])
    step(rows=0)
    join = lambda **kw: sp.linear_attention_join(**{**dict(P=4, heads=2, key_size=64, value_size=32, gathered=A[0],  # noqa: E731
                                                           out=A[1]), **kw})
    refused(sp.ERR_ARG, join, P=0, n_ranks=1)
    refused(sp.ERR_ARG, join, first_rank=2, n_ranks=3)
    refused(sp.ERR_ARG, join, gathered=None)
    refused(sp.ERR_LIMIT, join, value_size=129)
    refused(sp.ERR_ALIAS, join, out=A[0] + 64)
    refused(sp.ERR_ALIAS, join, first=A[1])
    refused(sp.ERR_OVERFLOW, join, P=1 << 30, first_rank=0, n_ranks=65535)


def test_norm_refusals():
    refused(sp.ERR_ARG, sp.NormPlan, 0)
    refused(sp.ERR_ARG, sp.NormPlan, 64, 9)
    refused(sp.ERR_ARG, sp.NormPlan, 64, sp.BF16, sp.F16)
    refused(sp.ERR_ARG, sp.NormPlan, 64, block=16)
    refused(sp.ERR_ARG, sp.NormPlan, 64, eps=0.0)
    refused(sp.ERR_ARG, sp.NormPlan, 64, eps=float("nan"))
    refused(sp.ERR_ARG, sp.NormPlan, 64, eps=float("inf"))
    refused(sp.ERR_LIMIT, sp.NormPlan, sp.NORM_MAX_WIDTH + 1)
    plan = sp.NormPlan(64, sp.BF16, block=32)
    refused(sp.ERR_WORKSPACE, plan.set_workspace, A[0], 8)
    forward = lambda **kw: plan.forward(**{**dict(rows=10, x=A[0], weight=A[1], residual=A[2], sum=A[3], y=A[4], y8=A[5],  # noqa: E731
                                                  scales=A[6], rstd=A[7]), **kw})
    refused(sp.ERR_ARG, forward, x=None)
    refused(sp.ERR_ARG, forward, scales=None)
    refused(sp.ERR_ARG, forward, y8=None)
    refused(sp.ERR_ARG, forward, y_ld=63)
    refused(sp.ERR_LIMIT, forward, rows=1 << 31)
    refused(sp.ERR_ALIAS, forward, y=A[0])
    refused(sp.ERR_ALIAS, forward, y=A[3])
    refused(sp.ERR_ALIAS, forward, sum=A[0] + 2)
    refused(sp.ERR_ALIAS, forward, sum=A[0], x_ld=64, sum_ld=65)
    refused(sp.ERR_ALIAS, forward, rstd=A[6] + 4)
    refused(sp.ERR_ALIAS, forward, scales=A[1])
    plan.forward(0, None, None)
    backward = lambda **kw: plan.backward(**{**dict(rows=10, dy=A[0], sum=A[1], weight=A[2], rstd=A[3], dx=A[4],  # noqa: E731
                                                    dweight=A[5], dsum=A[6]), **kw})
    refused(sp.ERR_WORKSPACE, backward)
    refused(sp.ERR_ARG, backward, rstd=None)
    refused(sp.ERR_ARG, backward, dx=None)
    refused(sp.ERR_ARG, backward, dsum_ld=2)
    refused(sp.ERR_ALIAS, backward, dx=A[1])
    refused(sp.ERR_ALIAS, backward, dx=A[0] + 2)
    refused(sp.ERR_ALIAS, backward, dweight=A[4])
    refused(sp.ERR_ALIAS, backward, dweight=A[2])


def test_clip_refusals():
    refused(sp.ERR_ARG, sp.ClipPlan, [], [])
    refused(sp.ERR_ARG, sp.ClipPlan, [4], [8])
    refused(sp.ERR_ARG, sp.ClipPlan, [4], [sp.F32], n_ranks=0)
    refused(sp.ERR_ARG, sp.ClipPlan, [4, 4], [sp.F32] * 2, ranks=[0, 2], n_ranks=2)
    refused(sp.ERR_LIMIT, sp.ClipPlan, [4], [sp.F32], n_ranks=65536)
    refused(sp.ERR_OVERFLOW, sp.ClipPlan, [1 << 50, 1], [sp.F32] * 2)
    refused(sp.ERR_LIMIT, sp.ClipPlan, [1 << 45, 16384], [sp.F32] * 2)
    with pytest.raises(ValueError):
        sp.ClipPlan([4], [sp.F32, sp.F32])
    with pytest.raises(ValueError):
        sp.ClipPlan([4], [sp.F32], ranks=[0, 0])
    plan = sp.ClipPlan([100, 0, 50], [sp.F32, sp.BF16, sp.F16])
    refused(sp.ERR_WORKSPACE, plan.set_workspace, A[0], 8)
    refused(sp.ERR_WORKSPACE, plan.set_tensors, A[:3], A[3:6])
    refused(sp.ERR_WORKSPACE, plan.set_tensors, A[:3], A[:3])
    refused(sp.ERR_WORKSPACE, plan.set_tensors, [A[0], None, A[2]])
    refused(sp.ERR_ARG, plan.set_tensors, [None, A[1], A[2]])
    refused(sp.ERR_ARG, plan.set_tensors, [A[0] + 2, A[1], A[2]])
    refused(sp.ERR_ARG, plan.set_tensors, A[:3], [A[3], A[4], A[5] + 1])
    refused(sp.ERR_ALIAS, plan.set_tensors, A[:3], [A[3], A[4], A[3] + 396])
    refused(sp.ERR_ALIAS, plan.set_tensors, A[:3], [A[0] + 4, A[4], A[5]])
    refused(sp.ERR_ALIAS, plan.set_tensors, A[:3], [A[2] + 96, A[4], A[5]])
    refused(sp.ERR_ALIAS, plan.set_tensors, [A[0], A[1], A[0] + 200], [A[0], A[4], A[5]])
    with pytest.raises(ValueError):
        plan.set_tensors(A[:2])
    with pytest.raises(TypeError):
        plan.set_tensors([OnTheGpu((100,), torch.bfloat16), OnTheGpu((0,), torch.bfloat16), OnTheGpu((50,), torch.float16)])
    refused(sp.ERR_WORKSPACE, plan.sums, A[0])
    refused(sp.ERR_ARG, plan.sums, None)
    refused(sp.ERR_WORKSPACE, plan.scale, A[0], 1, 1.0, A[1])
    refused(sp.ERR_ARG, plan.scale, A[0], 0, 1.0, A[1])
    refused(sp.ERR_ARG, plan.scale, A[0], 1, -1.0, A[1])
    refused(sp.ERR_ARG, plan.scale, A[0], 1, float("nan"), A[1])
    refused(sp.ERR_ARG, plan.scale, A[0], 1, 1.0, A[1], eps=-1.0)
    refused(sp.ERR_ALIAS, plan.scale, A[0], 1, 1.0, A[0])


BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("wrong", ["q", "k", "v", "log_decay", "o", "first", "summary"])
def test_linear_attention_takes_its_own_types(wrong):
    plan = sp.LinearAttentionPlan([128], 2, 64, 64)
    kinds = dict(q=((128, 128), BF), k=((128, 128), BF), v=((128, 128), BF), log_decay=((2,), F), o=((128, 128), BF),
                 first=((1, 2, 64, 64), F), summary=((1, 2 * 4097), F))
    good = {k: OnTheGpu(*v, address=(i + 1) << 40) for i, (k, v) in enumerate(kinds.items())}
    refused(sp.ERR_WORKSPACE, lambda: plan.forward(**good))
    shape, t = kinds[wrong]
    with pytest.raises(TypeError):
        plan.forward(**{**good, wrong: OnTheGpu(shape, torch.float16)})
    with pytest.raises(TypeError):
        plan.forward(**{**good, wrong: torch.zeros(shape, dtype=t)})
    with pytest.raises(ValueError):
        plan.forward(**{**good, wrong: OnTheGpu(shape, t, pitch=shape[-1] + 8)})


def test_norm_and_clip_take_their_own_types():
    plan = sp.NormPlan(64, sp.BF16, weight_dtype=sp.F32)
    x, w = OnTheGpu((10, 64), BF), OnTheGpu((64,), F, address=2 << 40)
    with pytest.raises(TypeError):
        plan.forward(10, x, OnTheGpu((64,), BF), y=x)
    with pytest.raises(TypeError):
        plan.forward(10, x, w, y8=OnTheGpu((10, 64), torch.float32), scales=OnTheGpu((10,), F))
    for t in (torch.uint8, torch.float8_e4m3fn):  # scales over x: refused after the types are found right
        refused(sp.ERR_ALIAS, plan.forward, 10, x, w, y8=OnTheGpu((10, 64), t, address=3 << 40), scales=OnTheGpu((10,), F))
    clip = sp.ClipPlan([4], [sp.F32])
    with pytest.raises(TypeError):
        clip.sums(OnTheGpu((1,), F))
    with pytest.raises(TypeError):
        clip.scale(OnTheGpu((1,), F), 1, 1.0, OnTheGpu((1, 2), F))


def test_linear_attention_keeps_states_of_cut_sequences_only():
    whole = sp.LinearAttentionPlan([64] * 3000, 4, 128, 128)
    assert whole.workspace_bytes < 1 << 20
    cut = sp.LinearAttentionPlan([64] * 3000 + [200000], 4, 128, 128)
    state = 4 * 128 * 128 * 4
    assert cut.workspace_bytes < 2 * state * (200000 // 128 + 1) + (1 << 20)
