"""Views that no row stride describes, no GPU: a row's elements follow one another (a head's and the heads), and the rows lie
equally far apart through all of a tensor's leading sizes.  Anything else is refused before an address is handed over
(the tensors here only look as if they lay on a GPU, and a call without a workspace is refused).  Which stride is given is
the caller's word."""
import pytest
import torch

import paper_2109_08751_b200 as sp
from test_train_host import refused

BF, F = torch.bfloat16, torch.float32


class OnTheGpu:
    """A view as the binding sees one: sizes and strides of a tensor without memory."""

    is_cuda = True

    def __init__(self, view, address):
        self.dtype, self.shape, self.address, self.view = view.dtype, view.shape, address, view

    def data_ptr(self):
        return self.address

    def stride(self, dim=None):
        return self.view.stride() if dim is None else self.view.stride(dim)

    def is_contiguous(self):
        return self.view.is_contiguous()


def new(*shape, dtype=BF):
    return torch.empty(*shape, dtype=dtype, device="meta")


def at(**views):
    return {k: OnTheGpu(v, (i + 1) << 40) for i, (k, v) in enumerate(views.items())}


T, H, D = 128, 4, 64
GOOD = {  # a tensor of T rows of H x D, and its row stride
    "dense": (new(T, H, D), H * D),
    "part of a wider row": (new(T, 3 * H * D)[:, H * D:2 * H * D], 3 * H * D),
    "part of a wider row, heads": (new(T, 3 * H * D)[:, :H * D].unflatten(1, (H, D)), 3 * H * D),
    "in a batch": (new(2, T // 2, 3, H, D)[:, :, 1], 3 * H * D),
    "every other row": (new(2 * T, H, D)[::2], 2 * H * D),
    "of one row's size only": (new(1, 5, H, D)[:, 2:3], 99999),
    "every third part of a wider row": (new(T, 6 * H * D)[:, :H * D], 2 * H * D),
    "a base that the stride takes rows from": (new(T, 3 * H * D), 3 * H * D),
}
BAD = {
    "heads of q, k and v by turns": (new(T, H, 3 * D)[:, :, :D], 3 * H * D),
    "heads before rows": (new(H, T, D).transpose(0, 1), D),
    "sizes before heads": (new(T, D, H).transpose(1, 2), H * D),
    "one head for all": (new(T, 1, D).expand(T, H, D), D),
    "one column for all": (new(T, H, 1).expand(T, H, D), H),
    "rows turned round": (new(H * D, T).T, H * D),
    "a padded batch": (new(2, T, H, D)[:, :T // 2 + 1], H * D),
}


def plan():
    return sp.LinearAttentionPlan([T], H, D, D)


@pytest.mark.parametrize("name", list(GOOD))
def test_views_that_a_row_stride_describes(name):
    v, ld = GOOD[name]
    dense = new(T, H, D)
    for x in ("q", "k", "v", "o"):
        given = at(**{**dict(q=dense, k=dense, v=dense, o=dense), x: v})
        refused(sp.ERR_WORKSPACE, lambda: plan().forward(log_decay=1 << 50, **given, **{x + "_ld": ld}))


@pytest.mark.parametrize("name", list(BAD))
def test_views_that_it_does_not_describe(name):
    v, ld = BAD[name]
    dense = new(T, H, D)
    for x in ("q", "k", "v", "o"):
        given = at(**{**dict(q=dense, k=dense, v=dense, o=dense), x: v})
        with pytest.raises(ValueError):
            plan().forward(log_decay=1 << 50, **given, **{x + "_ld": ld})
        # single tokens: nothing is launched, there are no slots and a negative count of them is refused
        with pytest.raises(ValueError):
            sp.linear_attention_step(T, H, D, D, sp.BF16, log_decay=1 << 50, state_in=1 << 51, state_out=1 << 51, n_slots=1, **given,
                                     **{x + "_ld": ld})
    for x in ("q", "k", "v", "do", "dq", "dk", "dv"):
        given = at(**{**{n: dense for n in ("q", "k", "v", "do", "dq", "dk", "dv")}, x: v})
        with pytest.raises(ValueError):
            plan().backward(log_decay=1 << 50, **given, **{x + "_ld": ld})


@pytest.mark.parametrize("name", list(BAD))
def test_the_other_operators_look_at_their_rows_too(name):
    v, ld = BAD[name]
    width = H * D
    scan, router, norm = sp.ScanPlan([T], width), sp.RouterPlan([T], width, 4), sp.NormPlan(width)
    a = at(**{x: new(T, width) for x in "abc"} | dict(v=v, i=new(T, 4, dtype=torch.int32), w=new(T, 4, dtype=F), e=new(T, dtype=F),
                                                      n=new(1, width + 1, dtype=torch.int32), s=new(1, width + 1, dtype=F),
                                                      state=new(T, width, dtype=F)))
    x, i, w, e, n, s = (a[k] for k in ("a", "i", "w", "e", "n", "s"))
    calls = [lambda: scan.forward(a["v"], x, a["b"], gate_ld=ld), lambda: scan.forward(x, a["v"], a["b"], x_ld=ld),
             lambda: scan.forward(x, a["b"], a["v"], y_ld=ld), lambda: router.forward(a["v"], i, w, e, n, s, ld=ld),
             lambda: router.backward(x, i, w, e, n, 1, a["v"], dlogits_ld=ld),
             lambda: sp.scan_step(T, width, sp.BF16, a["v"], x, a["state"], a["state"], a["b"], n_slots=1, gate_ld=ld),
             lambda: sp.scan_step(T, width, sp.BF16, x, a["v"], a["state"], a["state"], a["b"], n_slots=1, x_ld=ld),
             lambda: sp.scan_step(T, width, sp.BF16, x, a["b"], a["state"], a["state"], a["v"], n_slots=1, y_ld=ld),
             lambda: norm.forward(T, a["v"], y=x, x_ld=ld), lambda: norm.forward(T, x, y=a["v"], y_ld=ld),
             lambda: norm.backward(T, x, a["v"], None, e, a["b"], sum_ld=ld)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_states_and_matrices():
    x = new(6, 16)
    a = at(gate=x, x=x, y=x, wide=new(9, 64, dtype=F)[:, ::4], good=new(9, 64, dtype=F)[:, :16], turned=new(16, 9, dtype=F).T)
    step = lambda s, ld: sp.scan_step(6, 16, sp.BF16, a["gate"], a["x"], s, s, a["y"], n_slots=1, state_ld=ld)  # noqa: E731
    refused(sp.ERR_ARG, step, a["good"], 64)  # fewer slots than rows
    for s, ld in (("wide", 64), ("turned", 16)):
        with pytest.raises(ValueError):
            step(a[s], ld)
    plan = sp.OrthoPlan(3, 8, 16)
    b = at(one=new(3, 8, 16), beside=new(8, 3, 16), out=new(3, 8, 16), turned=new(3, 16, 8).transpose(1, 2), m=new(3, 8, 16, dtype=F),
           mt=new(3, 16, 8, dtype=F).transpose(1, 2))
    ortho = lambda v, **kw: plan.orthogonalize(v, b["out"], **kw)  # noqa: E731
    refused(sp.ERR_WORKSPACE, ortho, b["one"], ld=16, stride=128)
    refused(sp.ERR_WORKSPACE, ortho, b["beside"], ld=48, stride=16)
    refused(sp.ERR_WORKSPACE, ortho, OnTheGpu(new(8, 3, 16).transpose(0, 1), 7 << 40), ld=48, stride=16)
    with pytest.raises(ValueError):
        ortho(b["turned"], ld=16, stride=128)
    for wrong in ("momentum", "weight"):
        for side in ("in", "out"):
            given = dict(momentum_in=b["m"], momentum_out=b["m"], weight_in=b["m"], weight_out=b["m"])
            with pytest.raises(ValueError):
                plan.muon_step(b["one"], **{**given, f"{wrong}_{side}": b["mt"]}, weight_dtype=sp.F32, lr=0.1, momentum_ld=16,
                               weight_ld=16)
