"""What the binding of the training operators makes sure of before it hands over addresses, no GPU: tensors lie in
device memory, have the operator's type, and rows with gaps come with their stride.  The tensors here only look
as if they lay on a GPU (nothing reads them: every call is refused, at the latest for want of a workspace)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2109_08751_b200 as sp


class OnTheGpu:
    """A tensor as the binding sees one."""

    is_cuda = True

    def __init__(self, shape, dtype=torch.float32, address=1 << 40, pitch=None):
        self.dtype, self.address = dtype, address
        self.gaps = pitch is not None and pitch != shape[-1]

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return not self.gaps


BF, F, I, B = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def tensors(**kinds):
    """name: (shape, dtype) or None -> tensors at addresses of their own."""
    return {k: None if v is None else OnTheGpu(*v, address=(i + 1) << 40) for i, (k, v) in enumerate(kinds.items())}


SCAN, ROUTER, ORTHO = lambda: sp.ScanPlan([100, 28], 16, sp.BF16), lambda: sp.RouterPlan([100], 64, 4), \
    lambda: sp.OrthoPlan(1, 64, 96)
#: plan and call, its tensors, those among them that have a row stride (its argument), other arguments
CALLS = {
    "scan forward": (SCAN, "forward", dict(gate=((128, 16), BF), x=((128, 16), BF), y=((128, 16), BF), h0=((2, 16), F),
                                           summary=((2, 2, 16), F), carry=((2, 16), F)),
                     dict(gate="gate_ld", x="x_ld", y="y_ld", h0="h0_ld"), {}),
    "scan backward": (SCAN, "backward", dict(gate=((128, 16), BF), x=((128, 16), BF), carry=((2, 16), F), dy=((128, 16), BF),
                                             dgate=((128, 16), BF), dx=((128, 16), BF), dlast=((2, 16), F),
                                             dsummary=((2, 2, 16), F)),
                      dict(gate="gate_ld", x="x_ld", dy="dy_ld", dgate="dgate_ld", dx="dx_ld", dlast="dlast_ld"), {}),
    "router forward": (ROUTER, "forward", dict(logits=((100, 64), BF), indices=((100, 4), I), weights=((100, 4), F),
                                               lse=((100,), F), counts=((1, 65), I), sums=((1, 65), F), mask=((100,), B)),
                       dict(logits="ld"), {}),
    "router backward": (ROUTER, "backward", dict(logits=((100, 64), BF), indices=((100, 4), I), weights=((100, 4), F),
                                                 lse=((100,), F), gathered=((1, 65), I), dlogits=((100, 64), BF),
                                                 dweights=((100, 4), F), dloss=((1,), F), mask=((100,), torch.bool)),
                        dict(logits="ld", dlogits="dlogits_ld"), dict(G=1)),
    "orthogonalize": (ORTHO, "orthogonalize", dict(update=((64, 96), BF), out=((64, 96), BF)),
                      dict(update="ld", out="out_ld"), {}),
    "muon step": (ORTHO, "muon_step", dict(grad=((64, 96), BF), momentum_in=((64, 96), F), momentum_out=((64, 96), F),
                                           weight_in=((64, 96), torch.float16), weight_out=((64, 96), torch.float16)),
                  dict(grad="grad_ld", momentum_in="momentum_ld", momentum_out="momentum_ld", weight_in="weight_ld",
                       weight_out="weight_ld"), dict(weight_dtype=sp.F16, lr=0.1)),
    "single tokens": (None, "scan_step", dict(gate=((4, 8), BF), x=((4, 8), BF), state_in=((9, 8), F), state_out=((9, 8), F),
                                              y=((4, 8), BF), slots=((4,), I)),
                      dict(gate="gate_ld", x="x_ld", y="y_ld", state_in="state_ld", state_out="state_ld"),
                      dict(rows=4, channels=8, dtype=sp.BF16, n_slots=-1)),
    "join": (None, "scan_join", dict(gathered=((4, 4, 2, 8), F), out=((4, 8), F), h0=((8,), F)), dict(out="out_ld"),
             dict(P=4, channels=8, first_rank=7)),
    "balance": (ROUTER, "balance", dict(gathered=((1, 65), I), sums=((1, 65), F), loss=((1,), F)), {}, dict(G=0, alpha=1.0)),
}


def case(name):
    make, method, kinds, strided, other = CALLS[name]
    return getattr(make() if make else sp, method), kinds, strided, other


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_as_they_should_be_reach_the_library(name):
    call, kinds, strided, other = case(name)
    with pytest.raises(sp.SparbitError):    # no workspace, or the argument that is wrong on purpose
        call(**tensors(**kinds), **other)


@pytest.mark.parametrize("name", list(CALLS))
def test_host_memory_and_other_types_are_refused(name):
    call, kinds, _, other = case(name)
    for which, (shape, dtype) in kinds.items():
        with pytest.raises(TypeError):
            call(**{**tensors(**kinds), which: torch.zeros(shape, dtype=dtype)}, **other)
        if which == "carry":    # bytes, whatever their type
            continue
        for wrong in (BF, torch.float16, F, I, B, torch.float64, torch.int64):
            if wrong != dtype and not (dtype == torch.bool and wrong == B):
                with pytest.raises(TypeError):
                    call(**{**tensors(**kinds), which: OnTheGpu(shape, wrong)}, **other)


@pytest.mark.parametrize("name", list(CALLS))
def test_gaps_between_rows_need_their_stride(name):
    call, kinds, strided, other = case(name)
    for which, (shape, dtype) in kinds.items():
        given = {**tensors(**kinds), which: OnTheGpu(shape, dtype, 99 << 40, pitch=shape[-1] + 24)}
        with pytest.raises(ValueError):
            call(**given, **other)
        if which in strided:
            with pytest.raises(sp.SparbitError):
                call(**given, **other, **{strided[which]: shape[-1] + 24})


@pytest.mark.parametrize("name", [n for n in CALLS if CALLS[n][2]])
def test_a_row_stride_of_zero_is_not_the_default(name):
    call, kinds, strided, other = case(name)
    if name == "single tokens":
        other = dict(other, n_slots=9)
    elif name == "join":
        other = dict(other, first_rank=0)
    for argument in set(strided.values()):
        with pytest.raises(sp.SparbitError) as e:
            call(**tensors(**kinds), **other, **{argument: 0})
        assert e.value.code == sp.ERR_ARG, argument


def test_a_workspace_on_the_host_is_refused():
    for make in (SCAN, ROUTER, ORTHO):
        plan = make()
        with pytest.raises(TypeError):
            plan.set_workspace(torch.zeros(plan.workspace_bytes, dtype=B), plan.workspace_bytes)


def test_sizes_may_be_numpy_integers():
    """Whatever behaves like an int is a size, in the calls that convert ints the fast way too."""
    call, kinds, strided, other = case("single tokens")
    n = np.int64
    with pytest.raises(sp.SparbitError) as e:
        call(**{**tensors(**kinds), **other, "slots": None, **dict(rows=n(4), channels=n(8), n_slots=n(2), gate_ld=n(8))})
    assert e.value.code == sp.ERR_ARG
    call, kinds, strided, other = case("router forward")
    with pytest.raises(sp.SparbitError) as e:
        call(**tensors(**kinds), ld=n(64))
    assert e.value.code == sp.ERR_WORKSPACE
    with pytest.raises(ctypes.ArgumentError):
        call(**tensors(**kinds), ld=64.0)


class Address:
    """Something that has an address and says nothing else of itself."""

    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("name", list(CALLS))
def test_what_is_no_tensor_is_taken_as_it_is(name):
    """Numbers, numpy arrays and anything else with data_ptr(): the caller's word, as the library's other calls take it."""
    call, kinds, strided, other = case(name)
    for make in (Address, int, lambda a: np.empty(64, np.uint8)):
        given = {k: make((i + 1) << 40) for i, k in enumerate(kinds)}
        with pytest.raises(sp.SparbitError):
            call(**given, **other)
