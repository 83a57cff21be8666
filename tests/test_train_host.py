"""Host side of the training operators (include/sparbit_train.h), no GPU: the header and the binding
name the same things, plans are made and refused as documented, and every argument error is found
before anything is launched (the addresses here are numbers that nothing reads)."""
import ctypes
import re
import subprocess
from pathlib import Path

import pytest

import paper_2109_08751_b200 as sp
from paper_2109_08751_b200 import train

ROOT = Path(__file__).resolve().parent.parent
GPU_SIZED = 1 << 40  # addresses far apart from one another


def header():
    text = (ROOT / "include" / "sparbit_train.h").read_text()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_binding_names_what_the_header_declares():
    declared = set(re.findall(r"\b(sparbit_[a-z_]+)\s*\(", header()))
    assert declared == set(train.SYMBOLS), declared ^ set(train.SYMBOLS)
    lib = ctypes.CDLL(str(ROOT / "paper_2109_08751_b200" / "libsparbit_b200.so"))
    for name in declared:
        assert hasattr(lib, name), name


def test_binding_constants_match_the_header():
    for body in re.findall(r"enum\s*\{(.*?)\}", header(), flags=re.S):
        for name, value in re.findall(r"SPARBIT_([A-Z0-9_]+)\s*=\s*(-?\d+)", body):
            assert getattr(sp, name) == int(value), name
    for name, value in re.findall(r"#define SPARBIT_([A-Z0-9_]+) (\d+)", header()):
        assert getattr(sp, name) == int(value), name


def test_header_is_plain_c(tmp_path):
    source = tmp_path / "t.c"
    source.write_text('#include "sparbit_train.h"\nint main(void) { return sparbit_scan_plan_destroy(0); }\n')
    exe = tmp_path / "t"
    lib = ROOT / "paper_2109_08751_b200"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", f"-I{ROOT / 'include'}", str(source),
                    "-o", str(exe), f"-L{lib}", "-lsparbit_b200", f"-Wl,-rpath,{lib}"], check=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


def refused(code, call, *args, **kw):
    with pytest.raises(sp.SparbitError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_scan_plan_refusals():
    refused(sp.ERR_ARG, sp.ScanPlan, [], 8)
    refused(sp.ERR_ARG, sp.ScanPlan, [4], 0)
    refused(sp.ERR_ARG, sp.ScanPlan, [4], 8, 7)
    refused(sp.ERR_LIMIT, sp.ScanPlan, [4], (1 << 20) + 1)
    refused(sp.ERR_OVERFLOW, sp.ScanPlan, [1 << 45, 1 << 45], 8)
    refused(sp.ERR_LIMIT, sp.ScanPlan, [1 << 40], 8)
    refused(sp.ERR_LIMIT, sp.ScanPlan, [0] * 65536, 8)
    plan = sp.ScanPlan([0, 1, 128, 129], 10)
    assert plan.carry_bytes == 4 * 10 * 4   # one state per started piece of 128 steps
    assert plan.workspace_bytes > 0
    plan.destroy()


def test_scan_call_refusals():
    plan = sp.ScanPlan([100, 28], 16, sp.BF16)
    a = [GPU_SIZED * (i + 1) for i in range(8)]
    refused(sp.ERR_WORKSPACE, plan.set_workspace, None, 1 << 20)
    refused(sp.ERR_WORKSPACE, plan.set_workspace, a[0], 16)
    refused(sp.ERR_WORKSPACE, plan.set_workspace, a[0] + 8, 1 << 30)
    refused(sp.ERR_WORKSPACE, plan.forward, a[0], a[1], a[2])       # none set yet
    refused(sp.ERR_ARG, plan.forward, None, a[1], a[2])
    refused(sp.ERR_ARG, plan.forward, a[0], None, a[2])
    refused(sp.ERR_ARG, plan.forward, a[0], a[1], a[2], gate_ld=15)
    refused(sp.ERR_ARG, plan.forward, a[0], a[1], a[2], h0=a[3], h0_ld=8)
    refused(sp.ERR_ALIAS, plan.forward, a[0], a[1], a[1])
    refused(sp.ERR_ALIAS, plan.forward, a[0], a[1], a[0] + 127 * 16 * 2 + 30)
    refused(sp.ERR_ALIAS, plan.forward, a[0], a[1], a[2], summary=a[2] + 2)
    refused(sp.ERR_ALIAS, plan.forward, a[0], a[1], a[2], summary=a[3], carry=a[3])
    # the halves of one buffer lie inside one address range without sharing a byte
    half = dict(gate_ld=32, x_ld=32)
    refused(sp.ERR_WORKSPACE, plan.forward, a[0], a[0] + 32, a[2], **half)
    refused(sp.ERR_WORKSPACE, plan.forward, a[0], a[1], a[0] + 32, gate_ld=32, y_ld=32)
    refused(sp.ERR_ALIAS, plan.forward, a[0], a[1], a[0] + 30, gate_ld=32, y_ld=32)
    refused(sp.ERR_ALIAS, plan.forward, a[0] + 32, a[1], a[0] + 2, gate_ld=32, y_ld=32)
    refused(sp.ERR_ARG, plan.backward, a[0], a[1], a[2], a[3], a[4], None)
    refused(sp.ERR_ARG, plan.backward, a[0], None, a[2], a[3], a[4], a[5])
    refused(sp.ERR_ARG, plan.backward, a[0], a[1], None, a[3], a[4], a[5])
    refused(sp.ERR_ALIAS, plan.backward, a[0], a[1], a[2], a[3], a[4], a[4])
    refused(sp.ERR_ALIAS, plan.backward, a[0], a[1], a[2], a[3], a[4], a[3])
    refused(sp.ERR_WORKSPACE, plan.backward, a[0], None, None, a[3], None, None, dsummary=a[6])


def test_scan_step_and_join_refusals():
    a = [GPU_SIZED * (i + 1) for i in range(8)]
    step = lambda **kw: sp.scan_step(**{**dict(rows=4, channels=8, dtype=sp.F32, gate=a[0], x=a[1], state_in=a[2],  # noqa: E731
                                               state_out=a[2], y=a[3]), **kw})
    refused(sp.ERR_ARG, step, channels=0)
    refused(sp.ERR_ARG, step, dtype=3)
    refused(sp.ERR_ARG, step, gate=None)
    refused(sp.ERR_ARG, step, n_slots=3)            # without slots every row needs its state
    refused(sp.ERR_ARG, step, state_out=None)
    refused(sp.ERR_ARG, step, state_ld=7)
    refused(sp.ERR_ALIAS, step, y=a[0])
    refused(sp.ERR_ALIAS, step, y=a[2] + 4 * 31)
    refused(sp.ERR_ALIAS, step, state_out=a[2] + 4)
    refused(sp.ERR_LIMIT, step, channels=(1 << 20) + 1)
    step(rows=0)                                    # nothing to do, nothing launched
    join = lambda **kw: sp.scan_join(**{**dict(P=4, channels=8, gathered=a[0], out=a[1]), **kw})  # noqa: E731
    refused(sp.ERR_ARG, join, P=0)
    refused(sp.ERR_ARG, join, first_rank=2, n_ranks=3)
    refused(sp.ERR_ARG, join, first_rank=-1, n_ranks=1)
    refused(sp.ERR_ARG, join, gathered=None)
    refused(sp.ERR_ARG, join, out_ld=4)
    refused(sp.ERR_ALIAS, join, out=a[0] + 64)


def test_router_refusals():
    refused(sp.ERR_ARG, sp.RouterPlan, [], 8, 2)
    refused(sp.ERR_ARG, sp.RouterPlan, [4], 8, 0)
    refused(sp.ERR_ARG, sp.RouterPlan, [4], 8, 9)
    refused(sp.ERR_ARG, sp.RouterPlan, [4], 8, 2, 5)
    refused(sp.ERR_LIMIT, sp.RouterPlan, [4], 1025, 2)
    refused(sp.ERR_LIMIT, sp.RouterPlan, [4], 64, 33)
    refused(sp.ERR_LIMIT, sp.RouterPlan, [1 << 30, 1 << 30], 64, 2)
    plan = sp.RouterPlan([100, 0, 5], 60, 4, sp.BF16)
    a = [GPU_SIZED * (i + 1) for i in range(12)]
    forward = lambda **kw: plan.forward(**{**dict(logits=a[0], indices=a[1], weights=a[2], lse=a[3], counts=a[4],  # noqa: E731
                                                  sums=a[5]), **kw})
    refused(sp.ERR_WORKSPACE, forward)
    refused(sp.ERR_ARG, forward, logits=None)
    refused(sp.ERR_ARG, forward, counts=None)
    refused(sp.ERR_ARG, forward, ld=59)
    refused(sp.ERR_ALIAS, forward, weights=a[1])
    refused(sp.ERR_ALIAS, forward, lse=a[0] + 2)
    refused(sp.ERR_ALIAS, forward, sums=a[4] + 3 * 61 * 4 - 1)
    backward = lambda **kw: plan.backward(**{**dict(logits=a[0], indices=a[1], weights=a[2], lse=a[3], gathered=a[4],  # noqa: E731
                                                    G=3, dlogits=a[6]), **kw})
    refused(sp.ERR_WORKSPACE, backward)
    refused(sp.ERR_ARG, backward, G=0)
    refused(sp.ERR_ARG, backward, gathered=None)
    refused(sp.ERR_ARG, backward, dlogits_ld=10)
    refused(sp.ERR_ALIAS, backward, dlogits=a[0])
    refused(sp.ERR_ARG, plan.balance, None, 3, a[1], a[2], alpha=1.0)
    refused(sp.ERR_ARG, plan.balance, a[0], 0, a[1], a[2], alpha=1.0)
    refused(sp.ERR_ALIAS, plan.balance, a[0], 3, a[1], a[1], alpha=1.0)


def test_ortho_refusals():
    refused(sp.ERR_ARG, sp.OrthoPlan, 0, 8, 8)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 0, 8)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, 9)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, sp.F32, steps=0)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, sp.F32, eps=-1.0)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, sp.F32, eps=float("nan"))
    refused(sp.ERR_LIMIT, sp.OrthoPlan, 1, 65537, 8)
    refused(sp.ERR_LIMIT, sp.OrthoPlan, 4097, 8, 8)
    refused(sp.ERR_LIMIT, sp.OrthoPlan, 1, 8, 8, steps=65)
    # an iteration that diverges, and one whose polynomial does not fit the operands
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, steps=3, coefficients=[(4.0, 4.0, 4.0)] * 3)
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, steps=1, coefficients=[(1.0, 300.0, -300.0)])
    refused(sp.ERR_ARG, sp.OrthoPlan, 1, 8, 8, steps=1, coefficients=[(float("nan"), 0.0, 0.0)])
    sp.OrthoPlan(1, 8, 8, steps=2, coefficients=[(1.875, -1.25, 0.375)] * 2).destroy()
    plan = sp.OrthoPlan(2, 64, 96, sp.BF16)
    refused(sp.ERR_ARG, plan.set_products, 2)
    a = [GPU_SIZED * (i + 1) for i in range(8)]
    refused(sp.ERR_WORKSPACE, plan.set_workspace, a[0], 1024)
    refused(sp.ERR_WORKSPACE, plan.orthogonalize, a[0], a[1])
    refused(sp.ERR_WORKSPACE, plan.status)
    refused(sp.ERR_ARG, plan.orthogonalize, None, a[1])
    refused(sp.ERR_ARG, plan.orthogonalize, a[0], a[1], ld=95)
    refused(sp.ERR_ARG, plan.orthogonalize, a[0], a[1], out_stride=64 * 96 - 1)
    refused(sp.ERR_ALIAS, plan.orthogonalize, a[0], a[0])
    refused(sp.ERR_ALIAS, plan.orthogonalize, a[0], a[0] + 2 * 64 * 96 * 2 - 2)
    refused(sp.ERR_WORKSPACE, plan.orthogonalize, a[0], a[0] + 96 * 2, ld=192, out_ld=192)   # side by side
    step = lambda **kw: plan.muon_step(**{**dict(grad=a[0], momentum_in=a[1], momentum_out=a[1], weight_in=a[2],  # noqa: E731
                                                 weight_out=a[2], weight_dtype=sp.F32, lr=0.1), **kw})
    refused(sp.ERR_WORKSPACE, step)
    refused(sp.ERR_ARG, step, weight_dtype=4)
    refused(sp.ERR_ARG, step, momentum_out=None)
    refused(sp.ERR_ARG, step, momentum_ld=90)
    refused(sp.ERR_ALIAS, step, momentum_out=a[2])
    refused(sp.ERR_ALIAS, step, weight_out=a[2] + 4)
    refused(sp.ERR_ALIAS, step, weight_out=a[0])
    with pytest.raises(ValueError):
        sp.OrthoPlan(1, 8, 8, steps=2, coefficients=[(1.0, 0.0, 0.0)])
