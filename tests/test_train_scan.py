"""The gated linear recurrence on the GPU against the formula in 64 bits.

Tolerances.  Every step of the recurrence rounds a few times to 24 bits, relative to values that no
state exceeds (M, the largest of |x|, |h0|): at most 16 units of 2^-24 M a step, over the gate, the
products, and the regrouping into pairs.  An error made at a step decays with the a_t after it, so
the error of a state is at most 16 * 2^-24 * M * w with w_t = a_t w_{t-1} + 1.  Rounding the result
to its type adds half a unit of that type.  Gradients follow the same recurrence against time.
"""
import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"f32": (sp.F32, torch.float32, 2.0 ** -24), "bf16": (sp.BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (sp.F16, torch.float16, 2.0 ** -11)}
STEP = 16 * 2.0 ** -24
TINY = 1e-7   # below this a 16-bit float is denormal; absolute


def dev(*shape, dtype=torch.float32, fill=None):
    t = torch.empty(*shape, dtype=dtype, device="cuda")
    return t if fill is None else t.fill_(fill)


def with_workspace(plan):
    ws = dev(max(1, plan.workspace_bytes), dtype=torch.uint8, fill=0xAB)
    plan.set_workspace(ws, ws.numel())
    return plan


def reference(gate, x, h0, dy, dlast):
    """One sequence in 64 bits: states, gradients, and the bounds of their errors."""
    T = gate.shape[0]
    a = torch.sigmoid(gate)
    keep = torch.sigmoid(-gate)
    h = torch.zeros(T + 1, gate.shape[1], dtype=torch.float64)
    h[0] = h0
    wh = torch.zeros_like(h)
    for t in range(T):
        h[t + 1] = a[t] * h[t] + keep[t] * x[t]
        wh[t + 1] = a[t] * wh[t] + 1
    c, g, wg = dlast.clone(), torch.zeros_like(x), torch.zeros_like(x)
    w = torch.zeros_like(dlast)
    for t in range(T - 1, -1, -1):
        g[t] = dy[t] + c
        w = w + 1
        wg[t] = w
        c = a[t] * g[t]
        w = a[t] * w
    M = max([1e-30] + [v.abs().max().item() for v in (x, h0) if v.numel()])
    MG = max([1e-30, g.abs().max().item() if T else 0.0, dlast.abs().max().item()])
    eh, eg = STEP * M * wh, STEP * MG * wg
    aa = a * keep
    dgate = g * (h[:-1] - x) * aa
    egate = aa * (g.abs() * eh[:-1] + eg * (h[:-1] - x).abs() + STEP * MG * M)
    return dict(h=h, eh=eh, dgate=dgate, egate=egate, dx=g * keep, ex=keep * (eg + STEP * MG), dh0=c,
                edh0=STEP * MG * (w + 1), decay=a.prod(0))


def close(got, want, bound, unit, what):
    err = (got.double().cpu() - want).abs()
    lim = bound + unit * want.abs() + TINY * 2.0 ** -24 + (6e-8 if unit > 2.0 ** -20 and unit < 2.0 ** -9 else 0.0)
    bad = ~(err <= lim)
    assert not bad.any(), (what, err[bad].max().item(), lim[bad].min().item(), int(bad.sum()))


def case(lengths, D, dtype, seed=0, mean=3.0, std=1.5):
    _, t, _ = TYPES[dtype]
    g = torch.Generator().manual_seed(seed)
    rows, n = sum(lengths), len(lengths)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(gate=(r(rows, D) * std + mean).to(t), x=r(rows, D).to(t), dy=(r(rows, D) * 0.1).to(t), h0=r(n, D),
                dlast=r(n, D))


def padded(v, pad, shift=0):
    """A device copy of v whose rows are `pad` elements further apart, `shift` elements into its buffer."""
    buf = torch.full((v.shape[0] * (v.shape[1] + pad) + shift + 1,), 7.0, dtype=v.dtype, device="cuda")
    view = buf[shift:shift + v.shape[0] * (v.shape[1] + pad)].view(v.shape[0], v.shape[1] + pad)[:, :v.shape[1]]
    view.copy_(v)
    return buf, view


def run_and_check(lengths, D, dtype, pad=0, shift=0, stream=None, **kw):
    code, t, unit = TYPES[dtype]
    c = case(lengths, D, dtype, **kw)
    plan = with_workspace(sp.ScanPlan(lengths, D, code))
    n, rows = len(lengths), sum(lengths)
    bufs = {k: padded(c[k], pad, shift) for k in ("gate", "x", "dy")}
    outs = {k: padded(torch.zeros(rows, D, dtype=t), pad, shift) for k in ("y", "dgate", "dx")}
    h0, dlast = c["h0"].cuda(), c["dlast"].cuda()
    summary, dsummary = dev(n, 2, D, fill=5), dev(n, 2, D, fill=5)
    carry = dev(plan.carry_bytes // 4 + 4, fill=9)
    ld = D + pad
    torch.cuda.synchronize()
    plan.forward(bufs["gate"][1], bufs["x"][1], outs["y"][1], h0=h0, summary=summary, carry=carry, gate_ld=ld, x_ld=ld,
                 y_ld=ld, stream=stream)
    plan.backward(bufs["gate"][1], bufs["x"][1], carry, bufs["dy"][1], outs["dgate"][1], outs["dx"][1], dlast=dlast,
                  dsummary=dsummary, gate_ld=ld, x_ld=ld, dy_ld=ld, dgate_ld=ld, dx_ld=ld, stream=stream)
    torch.cuda.synchronize()
    # nothing outside the rows was written
    for buf, view in outs.values():
        assert int((buf != 7.0).sum()) <= view.numel()
        rest = buf.clone()
        rest[shift:shift + rows * ld].view(rows, ld)[:, :D] = 7.0
        assert (rest == 7.0).all()
    assert (carry[plan.carry_bytes // 4:] == 9).all()
    at = 0
    for s, T in enumerate(lengths):
        part = slice(at, at + T)
        at += T
        w = reference(*(v.double() for v in (c["gate"][part], c["x"][part], c["h0"][s], c["dy"][part], c["dlast"][s])))
        close(outs["y"][1][part], w["h"][1:], w["eh"][1:], unit, f"y {s}")
        close(summary[s, 1], w["h"][-1], w["eh"][-1], 0, f"last {s}")
        close(summary[s, 0], w["decay"], STEP * max(1, T) * w["decay"] + 1e-37, 0, f"decay {s}")
        close(dsummary[s, 0], w["decay"], STEP * max(1, T) * w["decay"] + 1e-37, 0, f"decay back {s}")
        close(outs["dgate"][1][part], w["dgate"], w["egate"], unit, f"dgate {s}")
        close(outs["dx"][1][part], w["dx"], w["ex"], unit, f"dx {s}")
        close(dsummary[s, 1], w["dh0"], w["edh0"], 0, f"dh0 {s}")
    return plan


LENGTHS = [[1], [0], [0, 1, 0], [2, 3], [127], [128], [129], [255, 1, 256, 257], [1000, 0, 33], [4500]]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_lengths(lengths, dtype):
    run_and_check(lengths, 66, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [1, 2, 3, 8, 63, 64, 65, 128, 200, 260, 1000])
def test_channels(D, dtype):
    run_and_check([150, 7], D, dtype, seed=D)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D,pad,shift", [(64, 64, 0), (64, 2, 0), (64, 1, 0), (64, 0, 1), (64, 4, 2), (64, 8, 8), (63, 1, 0),
                                         (128, 8, 4)])
def test_strides_and_alignment(D, pad, shift, dtype):
    run_and_check([131, 5], D, dtype, pad=pad, shift=shift, seed=pad)


@pytest.mark.parametrize("mean,std", [(-5.0, 3.0), (0.0, 0.1), (9.0, 1.0), (0.0, 60.0)])
def test_gates_over_their_range(mean, std):
    """From gates that forget everything to gates that keep everything."""
    run_and_check([300, 1000], 64, "f32", mean=mean, std=std)
    run_and_check([300, 1000], 64, "bf16", mean=mean, std=std)


def test_many_short_sequences():
    run_and_check([i % 5 for i in range(300)], 48, "bf16")


def test_a_stream_of_ones_own():
    stream = torch.cuda.Stream()
    run_and_check([700, 20], 64, "bf16", stream=stream)


def test_same_plan_again_and_in_a_graph():
    code, t, _ = TYPES["bf16"]
    lengths, D = [3000, 500], 192
    plan = with_workspace(sp.ScanPlan(lengths, D, code))
    c = {k: v.cuda() for k, v in case(lengths, D, "bf16").items()}
    rows = sum(lengths)

    def buffers():
        return dict(y=dev(rows, D, dtype=t), carry=dev(plan.carry_bytes // 4), dgate=dev(rows, D, dtype=t),
                    dx=dev(rows, D, dtype=t), summary=dev(2, 2, D), dsummary=dev(2, 2, D))

    def call(b, stream):
        plan.forward(c["gate"], c["x"], b["y"], h0=c["h0"], summary=b["summary"], carry=b["carry"], stream=stream)
        plan.backward(c["gate"], c["x"], b["carry"], c["dy"], b["dgate"], b["dx"], dlast=c["dlast"],
                      dsummary=b["dsummary"], stream=stream)

    first, second = buffers(), buffers()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(first, stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(second, stream)
    for _ in range(20):
        for v in second.values():
            v.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], second[k]), k   # bit for bit: no order depends on timing


def test_summary_only_equals_the_full_pass():
    code, t, _ = TYPES["bf16"]
    lengths, D = [1, 0, 400, 129], 64
    plan = with_workspace(sp.ScanPlan(lengths, D, code))
    c = {k: v.cuda() for k, v in case(lengths, D, "bf16").items()}
    full, only = dev(4, 2, D), dev(4, 2, D)
    plan.forward(c["gate"], c["x"], dev(sum(lengths), D, dtype=t), summary=full)
    plan.forward(c["gate"], c["x"], None, summary=only)
    assert torch.equal(full, only)
    carry, dg, dx = dev(plan.carry_bytes // 4), dev(sum(lengths), D, dtype=t), dev(sum(lengths), D, dtype=t)
    plan.forward(c["gate"], c["x"], None, carry=carry)
    plan.backward(c["gate"], c["x"], carry, c["dy"], dg, dx, dsummary=full)
    plan.backward(c["gate"], None, None, c["dy"], None, None, dsummary=only)
    assert torch.equal(full, only)


def test_what_is_not_finite_stays_in_its_sequence_and_channel():
    code, t, unit = TYPES["f32"]
    lengths, D = [300, 300], 64
    c = case(lengths, D, "f32")
    c["gate"][10, 3], c["gate"][20, 4], c["x"][30, 5] = float("nan"), float("inf"), float("inf")
    c["gate"][40, 6], c["x"][40, 6] = float("-inf"), 2.5
    plan = with_workspace(sp.ScanPlan(lengths, D, code))
    y = dev(600, D)
    plan.forward(c["gate"].cuda(), c["x"].cuda(), y, h0=c["h0"].cuda())
    y = y.cpu()
    assert torch.isnan(y[10:300, 3]).all() and torch.isfinite(y[:10, 3]).all() and torch.isfinite(y[300:, 3]).all()
    assert torch.isinf(y[30:300, 5]).all() and torch.isfinite(y[300:, 5]).all()
    assert torch.equal(y[20, 4], y[19, 4])      # a = 1 keeps the state
    assert y[40, 6] == 2.5                      # a = 0 replaces it
    fine = [ch for ch in range(D) if ch not in (3, 5)]
    assert torch.isfinite(y[:, fine]).all()


def test_gradient_against_differences():
    """Directional derivative of the 64-bit forward formula against the library's gradients."""
    lengths, D = [200, 61], 32
    c = case(lengths, D, "f32", mean=1.0)
    plan = with_workspace(sp.ScanPlan(lengths, D, sp.F32))
    d = {k: v.cuda() for k, v in c.items()}
    y, dg, dx, ds = dev(261, D), dev(261, D), dev(261, D), dev(2, 2, D)
    carry = dev(plan.carry_bytes // 4)
    plan.forward(d["gate"], d["x"], y, h0=d["h0"], carry=carry)
    plan.backward(d["gate"], d["x"], carry, d["dy"], dg, dx, dlast=d["dlast"], dsummary=ds)
    gen = torch.Generator().manual_seed(5)
    for which, grad in (("gate", dg), ("x", dx), ("h0", ds[:, 1])):
        way = torch.randn(c[which].shape, generator=gen, dtype=torch.float64)

        def loss(eps):
            v = {k: t.double() for k, t in c.items()}
            v[which] = v[which] + eps * way
            total, at = 0.0, 0
            for s, T in enumerate(lengths):
                h = v["h0"][s]
                for t in range(at, at + T):
                    a = torch.sigmoid(v["gate"][t])
                    h = a * h + (1 - a) * v["x"][t]
                    total = total + (h * v["dy"][t]).sum()
                total = total + (h * v["dlast"][s]).sum()
                at += T
            return total.item()

        eps = 1e-4
        want = (loss(eps) - loss(-eps)) / (2 * eps)
        terms = grad.double().cpu() * way
        got = terms.sum().item()
        # third derivatives times eps^2, and the gradients' own rounding
        assert abs(got - want) <= 1e-5 * terms.abs().sum().item(), (which, got, want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,D", [(1, 1), (3, 64), (5, 63), (64, 4096), (2, 1000)])
def test_single_tokens(rows, D, dtype):
    code, t, unit = TYPES[dtype]
    c = case([rows], D, dtype, seed=rows)
    n_slots = rows + 3
    gen = torch.Generator().manual_seed(1)
    table = torch.randn(n_slots, D, generator=gen)
    slots = torch.randperm(n_slots, generator=gen)[:rows].to(torch.int32)
    if rows >= 3:
        slots[1], slots[2] = -1, n_slots + 7    # rows without a sequence
    a = torch.sigmoid(c["gate"].double())
    valid = (slots >= 0) & (slots < n_slots)
    want_state, want_y = table.double().clone(), torch.zeros(rows, D, dtype=torch.float64)
    for i in range(rows):
        if valid[i]:
            want_y[i] = a[i] * table[slots[i]].double() + torch.sigmoid(-c["gate"][i].double()) * c["x"][i].double()
            want_state[slots[i]] = want_y[i]
    y, out = dev(rows, D, dtype=t), table.cuda()
    other = table.cuda()
    for state_in, state_out in ((table.cuda(), other), (out, out)):
        sp.scan_step(rows, D, code, c["gate"].cuda(), c["x"].cuda(), state_in, state_out, y, slots=slots.cuda(),
                     n_slots=n_slots)
        M = max(table.abs().max().item(), c["x"].abs().max().item())
        close(state_out, want_state, STEP * M, 0, "state")
        close(y, want_y, STEP * M, unit, "y")
    sp.scan_step(rows, D, code, c["gate"].cuda(), c["x"].cuda(), table.cuda(), other, y)
    want = a * table[:rows].double() + torch.sigmoid(-c["gate"].double()) * c["x"].double()
    close(y, want, STEP * M, unit, "y without slots")


def test_prefill_then_tokens_equals_one_pass():
    """Serving: the states after a prompt, carried on one token at a time."""
    T, D, prompt = 40, 128, 33
    c = {k: v.cuda() for k, v in case([T], D, "f32").items()}
    whole = with_workspace(sp.ScanPlan([T], D, sp.F32))
    y = dev(T, D)
    whole.forward(c["gate"], c["x"], y, h0=c["h0"])
    plan = with_workspace(sp.ScanPlan([prompt], D, sp.F32))
    part, summary, token = dev(prompt, D), dev(1, 2, D), dev(1, D)
    plan.forward(c["gate"], c["x"], part, h0=c["h0"], summary=summary)
    state = summary[:, 1].contiguous()
    bound = STEP * T * max(c["x"].abs().max().item(), c["h0"].abs().max().item())
    for t in range(prompt, T):
        sp.scan_step(1, D, sp.F32, c["gate"][t], c["x"][t], state, state, token)
        assert (token[0] - y[t]).abs().max().item() <= bound
    assert (part - y[:prompt]).abs().max().item() <= bound


@pytest.mark.parametrize("P", [1, 2, 5, 8])
def test_divided_by_time_over_ranks(P):
    """Slices whose summaries the library's own allgather exchanges give what the whole sequence gives."""
    D = 96
    lengths = [(37 * (r + 1)) % 200 for r in range(P)]
    T = sum(lengths)
    c = case([T], D, "f32", seed=P)
    d = {k: v.cuda() for k, v in c.items()}
    want = reference(c["gate"].double(), c["x"].double(), c["h0"][0].double(), c["dy"].double(), c["dlast"][0].double())
    plan = with_workspace(sp.ScanPlan(lengths, D, sp.F32))
    gather = sp.Plan(P, 2 * D * 4)
    block, gathered = dev(P, 2, D), dev(P, P, 2, D)
    first, last = dev(P, D + 4, fill=0), dev(P, D)
    y, dg, dx, ds, carry = dev(T, D), dev(T, D), dev(T, D), dev(P, 2, D), dev(plan.carry_bytes // 4)
    plan.forward(d["gate"], d["x"], None, summary=block)
    gather.allgather(block, gathered)
    sp.scan_join(P, D, gathered, first, h0=d["h0"], out_ld=D + 4)
    plan.forward(d["gate"], d["x"], y, h0=first, h0_ld=D + 4, carry=carry)
    plan.backward(d["gate"], None, None, d["dy"], None, None, dsummary=block)
    gather.allgather(block, gathered)
    sp.scan_join(P, D, gathered, last, h0=d["dlast"], reverse=True)
    plan.backward(d["gate"], d["x"], carry, d["dy"], dg, dx, dlast=last, dsummary=ds)
    close(y, want["h"][1:], want["eh"][1:], 2.0 ** -24, "y")
    close(dg, want["dgate"], want["egate"], 2.0 ** -24, "dgate")
    close(dx, want["dx"], want["ex"], 2.0 ** -24, "dx")
    close(ds[0, 1], want["dh0"], want["edh0"], 0, "dh0")
    # one process that is rank r computes the same first state from its own receive buffer
    alone = dev(1, D)
    for r in range(P):
        sp.scan_join(P, D, gathered[r], alone, h0=d["dlast"], reverse=True, first_rank=r, n_ranks=1)
        assert torch.equal(alone[0], last[r])


def test_a_wait_that_runs_out_is_reported():
    """States withheld on purpose: the kernel gives up after the limit, says so, and works again afterwards."""
    plan = with_workspace(sp.ScanPlan([5000], 64, sp.BF16))
    c = {k: v.cuda() for k, v in case([5000], 64, "bf16").items()}
    y, again = dev(5000, 64, dtype=torch.bfloat16), dev(5000, 64, dtype=torch.bfloat16)
    plan.forward(c["gate"], c["x"], y)
    assert plan.status() == sp.OK
    plan.set_wait_test(True, 20_000_000)
    plan.forward(c["gate"], c["x"], again)
    assert plan.status() == sp.ERR_TIMEOUT
    plan.set_wait_test(False)
    plan.forward(c["gate"], c["x"], again)
    assert plan.status() == sp.OK and torch.equal(y, again)


def test_a_plan_without_workspace_or_on_no_buffer_is_refused():
    plan = sp.ScanPlan([10], 8, sp.F32)
    v = dev(10, 8)
    with pytest.raises(sp.SparbitError) as e:
        plan.forward(v, v, dev(10, 8))
    assert e.value.code == sp.ERR_WORKSPACE
