"""Measured cases of the training operators that stand next to the allgather.

Three operators of a training step whose state is divided over the ranks of a communicator, each with one
allgather in its middle: a gated linear recurrence over a sequence that is divided by time (the ranks exchange
what each slice does to a state), the router's choice of experts with its balance loss (the ranks exchange the
per-expert counts), and the orthogonalised update of a matrix (its rows are gathered first).

`run` computes them in elementary torch operations where `own` is false, in 32 bits with one rounding at the
end, and through the library where it is true.  `exact` has the same results in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
#: the quintic whose repetition drives every singular value towards one
QUINTIC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def listed():
    return [
        # one token for each of 48 running sequences, their states in a table of more slots: serving
        dict(name="scan_step_48", kind="scan_step", rows=48, slots=64, channels=4096, dtype="bf16"),
        # one prompt of an odd length, states only: prefill
        dict(name="scan_prompt_4097", kind="scan_forward", lengths="4097", channels=2048, dtype="bf16"),
        # packed documents of very different lengths, one of them empty and one a single token, in 32 bits
        dict(name="scan_packed_f32", kind="scan_train", lengths="1,0,777,3001,64,2500,129,5000", channels=1000,
             dtype="f32"),
        # an ordinary training batch: 8 sequences, forward and backward
        dict(name="scan_batch_train", kind="scan_train", lengths=",".join(["4096"] * 8), channels=2048,
             dtype="bf16"),
        # one long sequence divided over 8 ranks by time: summaries, their allgather, forward and backward
        dict(name="scan_sharded_long", kind="scan_sharded", lengths=",".join(["8192"] * 8), channels=2048,
             dtype="bf16"),
        # small square matrices, several at once: latency
        dict(name="ortho_small", kind="ortho", count=4, rows=256, cols=256, dtype="bf16", structure="random"),
        # odd and tall, as an embedding-side projection
        dict(name="ortho_tall_odd", kind="ortho", count=2, rows=3001, cols=1000, dtype="bf16", structure="lowrank"),
        # 32-bit gradients and weights of an attention projection
        dict(name="muon_f32", kind="muon", count=2, rows=1024, cols=4096, dtype="f32", structure="lowrank"),
        # the largest dense matrix of a step
        dict(name="muon_large", kind="muon", count=1, rows=4096, cols=8192, dtype="bf16", structure="decay"),
        # a short prompt through a router
        dict(name="router_prompt", kind="router_forward", tokens="200", experts=64, k=6, dtype="bf16", padding=0.0,
             renormalize=False),
        # 8 ranks with uneven numbers of tokens, some of them padding
        dict(name="router_train", kind="router_train", tokens="8192,8000,8192,7777,8192,1,8192,8192", experts=256,
             k=8, dtype="bf16", padding=0.1, renormalize=True),
        # few experts, 32-bit logits, many tokens
        dict(name="router_train_f32", kind="router_train", tokens=",".join(["32768"] * 4), experts=60, k=4,
             dtype="f32", padding=0.02, renormalize=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scan_step", "scan_forward", "scan_train", "scan_sharded", "ortho", "muon", "router_forward",
                       "router_train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "scan_step":
        rows = _log(rng, 1, 512)
        return dict(kind=kind, rows=rows, slots=rows + rng.randrange(0, 64), channels=_log(rng, 256, 8192), dtype=dtype)
    if kind.startswith("scan"):
        n = rng.randrange(2, 17) if kind == "scan_sharded" else _log(rng, 1, 16)
        channels = _log(rng, 128, 4096)
        most = max(64, min(65536, (1 << 27) // channels) // n)
        lengths = [_log(rng, 1, most) for _ in range(n)]
        return dict(kind=kind, lengths=",".join(map(str, lengths)), channels=channels, dtype=dtype)
    if kind in ("ortho", "muon"):
        rows, cols = _log(rng, 64, 4096), _log(rng, 64, 4096)
        most = max(1, min(8, (1 << 24) // (rows * cols)))
        return dict(kind=kind, count=rng.randrange(1, most + 1), rows=rows, cols=cols, dtype=dtype,
                    structure=rng.choice(["random", "lowrank", "decay"]))
    experts = _log(rng, 8, 512)
    n = 1 if kind == "router_forward" else rng.randrange(1, 9)
    most = max(16, (1 << 23) // experts // n)
    return dict(kind=kind, tokens=",".join(str(_log(rng, 1, most)) for _ in range(n)), experts=experts,
                k=rng.randrange(1, min(experts, 12) + 1), dtype=dtype,
                padding=rng.choice([0.0, 0.05, 0.5]), renormalize=rng.choice([True, False]))


def _ints(text):
    return [int(v) for v in text.split(",")]


def _inputs(case, seed):
    """The case's inputs on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["dtype"]]
    kind = case["kind"]

    def normal(*shape, mean=0.0, std=1.0, dtype=t):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean).to(dtype)

    s = dict(case=case, dtype=t)
    if kind == "scan_step":
        # the halves of one projection, so that each has a row stride of twice its width
        both = normal(case["rows"], 2 * case["channels"])
        both[:, :case["channels"]] += 3.0
        s["gate"], s["x"] = both[:, :case["channels"]], both[:, case["channels"]:]
        s["state"] = normal(case["slots"], case["channels"], std=0.3, dtype=torch.float32)
        s["slots"] = torch.randperm(case["slots"], generator=g, device="cuda")[:case["rows"]].to(torch.int32)
    elif kind.startswith("scan"):
        lengths = _ints(case["lengths"])
        rows, n, d = sum(lengths), len(lengths), case["channels"]
        # gates of a trained recurrence: most of them keep nearly all of the state
        s["gate"], s["x"] = normal(rows, d, mean=3.0, std=1.5), normal(rows, d)
        s["lengths"] = lengths
        if kind == "scan_sharded":
            s["h0"] = None
        else:
            s["h0"] = normal(n, d, std=0.3, dtype=torch.float32)
        if kind != "scan_forward":
            s["dy"] = normal(rows, d, std=1e-2)
            s["dlast"] = None if kind == "scan_sharded" else normal(n, d, std=1e-2, dtype=torch.float32)
    elif kind in ("ortho", "muon"):
        c, m, n = case["count"], case["rows"], case["cols"]
        if case["structure"] == "random":
            u = normal(c, m, n, std=1e-3, dtype=torch.float32)
        else:
            # what a gradient looks like: a product over fewer samples than dimensions, with or without decay
            r = max(1, min(m, n) // (8 if case["structure"] == "lowrank" else 1))
            left = normal(c, m, r, dtype=torch.float32)
            if case["structure"] == "decay":
                left /= torch.arange(1, r + 1, device="cuda", dtype=torch.float32)
            u = torch.bmm(left, normal(c, r, n, dtype=torch.float32)).mul_(1e-3 / math.sqrt(r))
            u += normal(c, m, n, std=2e-5, dtype=torch.float32)
        s["update"] = u.to(t)
        if kind == "muon":
            s["momentum"] = normal(c, m, n, std=5e-4, dtype=torch.float32)
            s["weight"] = normal(c, m, n, std=0.02)
    else:
        tokens, e = _ints(case["tokens"]), case["experts"]
        rows = sum(tokens)
        # some experts are liked more than others
        s["tokens"] = tokens
        s["logits"] = (normal(rows, e, dtype=torch.float32) + 0.5 * normal(e, dtype=torch.float32)).to(t)
        s["mask"] = (torch.rand(rows, generator=g, device="cuda") >= case["padding"]).to(torch.uint8)
        if case["padding"]:
            s["logits"][s["mask"] == 0] = float("nan")  # padding rows hold whatever was in the buffer
        s["dweights"] = normal(rows, case["k"], std=1e-2, dtype=torch.float32)
    return s


ALPHA, BETA = 1e-2, 1e-3  # weights of the balance and of the logit-size term
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2109_08751_b200 as sp

    kind, t = case["kind"], s["dtype"]
    code = {"f32": sp.F32, "bf16": sp.BF16, "f16": sp.F16}[case["dtype"]]
    s["sp"], s["code"] = sp, code

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def with_workspace(plan):
        s["plan"] = plan
        if plan.workspace_bytes:
            plan.set_workspace(empty(plan.workspace_bytes, dtype=torch.uint8), plan.workspace_bytes)

    if kind == "scan_step":
        s["y"], s["state_out"] = empty(case["rows"], case["channels"], dtype=t), s["state"].clone()
    elif kind.startswith("scan"):
        n, d, rows = len(s["lengths"]), case["channels"], sum(s["lengths"])
        with_workspace(sp.ScanPlan(s["lengths"], d, code))
        s["y"], s["summary"] = empty(rows, d, dtype=t), empty(n, 2, d)
        if kind != "scan_forward":
            s["carry"] = empty(s["plan"].carry_bytes, dtype=torch.uint8)
            s["dgate"], s["dx"], s["dsummary"] = empty(rows, d, dtype=t), empty(rows, d, dtype=t), empty(n, 2, d)
        if kind == "scan_sharded":
            s["gather"] = sp.Plan(n, 2 * d * 4)
            s["gathered"], s["h0"], s["dlast"] = empty(n, n, 2, d), empty(n, d), empty(n, d)
    elif kind in ("ortho", "muon"):
        with_workspace(sp.OrthoPlan(case["count"], case["rows"], case["cols"], code))
        if kind == "ortho":
            s["out"] = torch.empty_like(s["update"])
        else:
            s["momentum_out"], s["weight_out"] = torch.empty_like(s["momentum"]), torch.empty_like(s["weight"])
    else:
        n, e, k, rows = len(s["tokens"]), case["experts"], case["k"], sum(s["tokens"])
        with_workspace(sp.RouterPlan(s["tokens"], e, k, code, renormalize=case["renormalize"]))
        s["indices"], s["weights"], s["lse"] = empty(rows, k, dtype=torch.int32), empty(rows, k), empty(rows)
        s["counts"], s["sums"] = empty(n, e + 1, dtype=torch.int32), empty(n, e + 1)
        if kind == "router_train":
            s["gather"] = sp.Plan(n, (e + 1) * 4)
            s["gathered"], s["loss"] = empty(n, n, e + 1, dtype=torch.int32), empty(n)
            s["dlogits"] = torch.empty_like(s["logits"])
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---- through the library ---------------------------------------------------------------------------------


def _run_own(s):
    case, kind, sp = s["case"], s["case"]["kind"], s["sp"]
    plan = s.get("plan")
    stream = torch.cuda.current_stream()
    if kind == "scan_step":
        sp.scan_step(case["rows"], case["channels"], s["code"], s["gate"], s["x"], s["state"], s["state_out"], s["y"],
                     slots=s["slots"], n_slots=case["slots"], gate_ld=s["gate"].stride(0), x_ld=s["x"].stride(0),
                     stream=stream)
        return dict(y=s["y"], state=s["state_out"])
    if kind == "scan_forward":
        plan.forward(s["gate"], s["x"], s["y"], h0=s["h0"], summary=s["summary"], stream=stream)
        return dict(y=s["y"], last=s["summary"][:, 1])
    if kind == "scan_train":
        plan.forward(s["gate"], s["x"], s["y"], h0=s["h0"], summary=s["summary"], carry=s["carry"], stream=stream)
        plan.backward(s["gate"], s["x"], s["carry"], s["dy"], s["dgate"], s["dx"], dlast=s["dlast"],
                      dsummary=s["dsummary"], stream=stream)
        return dict(y=s["y"], last=s["summary"][:, 1], dgate=s["dgate"], dx=s["dx"], dh0=s["dsummary"][:, 1])
    if kind == "scan_sharded":
        # every rank's slice: what it does to a state; all ranks learn it; each works out where it starts
        plan.forward(s["gate"], s["x"], None, summary=s["summary"], stream=stream)
        s["gather"].allgather(s["summary"], s["gathered"], stream=stream)
        sp.scan_join(len(s["lengths"]), case["channels"], s["gathered"], s["h0"], stream=stream)
        plan.forward(s["gate"], s["x"], s["y"], h0=s["h0"], carry=s["carry"], stream=stream)
        # and the same against time for the gradient
        plan.backward(s["gate"], s["x"], None, s["dy"], None, None, dsummary=s["dsummary"], stream=stream)
        s["gather"].allgather(s["dsummary"], s["gathered"], stream=stream)
        sp.scan_join(len(s["lengths"]), case["channels"], s["gathered"], s["dlast"], reverse=True, stream=stream)
        plan.backward(s["gate"], s["x"], s["carry"], s["dy"], s["dgate"], s["dx"], dlast=s["dlast"], stream=stream)
        return dict(y=s["y"], dgate=s["dgate"], dx=s["dx"], h0=s["h0"], dlast=s["dlast"])
    if kind == "ortho":
        plan.orthogonalize(s["update"], s["out"], stream=stream)
        return s["out"]
    if kind == "muon":
        plan.muon_step(s["update"], s["momentum"], s["momentum_out"], s["weight"], s["weight_out"],
                       weight_dtype=s["code"], lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                       scale=_scale(case), stream=stream)
        return dict(weight=s["weight_out"], momentum=s["momentum_out"])
    plan.forward(s["logits"], s["indices"], s["weights"], s["lse"], s["counts"], s["sums"], mask=s["mask"],
                 stream=stream)
    out = dict(indices=s["indices"], weights=s["weights"], counts=s["counts"], sums=s["sums"])
    if kind == "router_forward":
        return out
    s["gather"].allgather(s["counts"], s["gathered"], stream=stream)
    ranks = len(s["tokens"])
    plan.balance(s["gathered"], ranks, s["sums"], s["loss"], alpha=ALPHA, beta=BETA, stream=stream)
    plan.backward(s["logits"], s["indices"], s["weights"], s["lse"], s["gathered"], ranks, s["dlogits"],
                  dweights=s["dweights"], alpha=ALPHA, beta=BETA, mask=s["mask"], stream=stream)
    return dict(out, loss=s["loss"], dlogits=s["dlogits"])


# ---- plain forms -----------------------------------------------------------------------------------------


def _scale(case):
    return 0.2 * math.sqrt(max(case["rows"], case["cols"]))


def _doubling(a, b):
    """Inclusive scan along the first axis of h_t = a_t h_{t-1} + b_t, by doubling the span that each row covers."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat([b[:d], torch.addcmul(b[d:], a[d:], b[:-d])])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return a, b


def _plain_scan(gate, x, h0):
    """The states and the decay of every step of one sequence, in 32 bits."""
    a = torch.sigmoid(gate)
    b = torch.sigmoid(-gate) * x
    total, h = _doubling(a, b)
    if h0 is not None:
        h = torch.addcmul(h, total, h0.expand_as(total))
    return a, h


def _plain_scan_back(gate, x, a, h, h0, dy, dlast):
    """Gradients of gate, x and the first state."""
    before = torch.cat([h0[None], h[:-1]])
    after = torch.cat([a[1:], torch.ones_like(a[:1])])  # what reaches step t from step t + 1
    g = dy.clone()
    g[-1] += dlast
    g = _doubling(after.flip(0), g.flip(0))[1].flip(0)
    keep = torch.sigmoid(-gate)
    return g * (before - x) * a * keep, g * keep, a[0] * g[0]


def _plain_ortho(u):
    """Five rounds of the quintic on u / |u|, in 32 bits."""
    tall = u.shape[-2] > u.shape[-1]
    x = u.transpose(-1, -2) if tall else u
    x = x / (x.square().sum((-1, -2), keepdim=True).sqrt() + EPS)
    a, b, c = QUINTIC
    for _ in range(5):
        gram = x @ x.transpose(-1, -2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(-1, -2) if tall else x


def _plain_router(s):
    case = s["case"]
    k, e = case["k"], case["experts"]
    valid = (s["mask"] != 0)[:, None]
    l = torch.where(valid, s["logits"].float(), 0.0)
    lse = torch.logsumexp(l, 1, keepdim=True)
    p = torch.exp(l - lse)
    order = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :k]
    chosen = p.gather(1, order)
    weights = chosen / chosen.sum(1, keepdim=True) if case["renormalize"] else chosen
    hit = torch.zeros_like(p).scatter_(1, order, 1.0) * valid
    count, total, at = [], [], 0
    for n in s["tokens"]:
        v = valid[at:at + n]
        count.append(torch.cat([hit[at:at + n].sum(0), v.sum()[None].float()]))
        z = (torch.where(v, lse[at:at + n], 0.0)).square().sum()[None]
        total.append(torch.cat([torch.where(v, p[at:at + n], 0.0).sum(0), z]))
        at += n
    out = dict(indices=torch.where(valid, order, -1).to(torch.int32), weights=torch.where(valid, weights, 0.0),
               counts=torch.stack(count).to(torch.int32), sums=torch.stack(total))
    if case["kind"] == "router_forward":
        return out
    everyone = out["counts"].sum(0).float()
    number = everyone[e].clamp_min(1)
    f = everyone[:e] / (number * k)
    out["loss"] = (ALPHA * e / number * (out["sums"][:, :e] * f).sum(1) + BETA / number * out["sums"][:, e])
    d = ALPHA * e / number * p * (f - (p * f).sum(1, keepdim=True)) + 2 * BETA / number * lse * p
    dw = s["dweights"]
    inner = (dw * weights).sum(1, keepdim=True)
    if case["renormalize"]:
        d = d.scatter_add(1, order, weights * (dw - inner))
    else:
        d = (d - p * inner).scatter_add(1, order, weights * dw)
    out["dlogits"] = torch.where(valid, d, 0.0).to(s["dtype"])
    return out


def _run_plain(s):
    case, kind, t = s["case"], s["case"]["kind"], s["dtype"]
    if kind == "scan_step":
        slots = s["slots"].long()
        g, x = s["gate"].float(), s["x"].float()
        h = torch.sigmoid(g) * s["state"][slots] + torch.sigmoid(-g) * x
        state = s["state"].clone()
        state[slots] = h
        return dict(y=h.to(t), state=state)
    if kind == "scan_sharded":
        # the slices make up one sequence
        zero = torch.zeros(case["channels"], device="cuda")
        gate, x, dy = s["gate"].float(), s["x"].float(), s["dy"].float()
        a, h = _plain_scan(gate, x, None)
        g_from = torch.cat([a[1:], torch.ones_like(a[:1])])
        g = _doubling(g_from.flip(0), dy.flip(0))[1].flip(0)
        before = torch.cat([zero[None], h[:-1]])
        keep = torch.sigmoid(-gate)
        at = torch.tensor(s["lengths"]).cumsum(0)[:-1].cuda()
        return dict(y=h.to(t), dgate=(g * (before - x) * a * keep).to(t), dx=(g * keep).to(t),
                    h0=torch.cat([zero[None], h[at - 1]]), dlast=torch.cat([(a * g)[at], zero[None]]))
    if kind.startswith("scan"):
        parts = {name: [] for name in ("y", "last", "dgate", "dx", "dh0")}
        at = 0
        for i, n in enumerate(s["lengths"]):
            h0 = s["h0"][i]
            if n == 0:
                parts["last"].append(h0)
                if kind == "scan_train":
                    parts["dh0"].append(s["dlast"][i])
                continue
            gate, x = s["gate"][at:at + n].float(), s["x"][at:at + n].float()
            a, h = _plain_scan(gate, x, h0)
            parts["y"].append(h.to(t))
            parts["last"].append(h[-1])
            if kind == "scan_train":
                dg, dx, dh = _plain_scan_back(gate, x, a, h, h0, s["dy"][at:at + n].float(), s["dlast"][i])
                parts["dgate"].append(dg.to(t))
                parts["dx"].append(dx.to(t))
                parts["dh0"].append(dh)
            at += n
        return {name: (torch.stack if name in ("last", "dh0") else torch.cat)(v) for name, v in parts.items() if v}
    if kind == "ortho":
        return _plain_ortho(s["update"].float()).to(t)
    if kind == "muon":
        g = s["update"].float()
        m = MOMENTUM * s["momentum"] + g
        x = _plain_ortho(g + MOMENTUM * m)
        w = (1 - LR * DECAY) * s["weight"].float() - LR * _scale(case) * x
        return dict(weight=w.to(t), momentum=m)
    return _plain_router(s)


# ---- 64 bits ---------------------------------------------------------------------------------------------


def _exact_scan(gate, x, h0, dy=None, dlast=None):
    """One sequence step by step."""
    gate, x = gate.double(), x.double()
    a = 1 / (1 + torch.exp(-gate))
    h = torch.empty(gate.shape[0] + 1, gate.shape[1], dtype=torch.float64, device="cuda")
    h[0] = h0
    b = x * (1 - a)
    for t in range(gate.shape[0]):
        torch.addcmul(b[t], a[t], h[t], out=h[t + 1])
    if dy is None:
        return h, None, None, None
    g = dy.double().clone()
    g[-1] += dlast
    for t in range(gate.shape[0] - 2, -1, -1):
        g[t].addcmul_(a[t + 1], g[t + 1])
    return h, g * (h[:-1] - x) * a * (1 - a), g * (1 - a), a * g


def _exact_ortho(u):
    u = u.double()
    u = u / (torch.linalg.matrix_norm(u) + EPS)[:, None, None]
    a, b, c = QUINTIC
    eye = torch.eye(min(u.shape[1:]), dtype=torch.float64, device="cuda")
    for _ in range(5):
        if u.shape[1] <= u.shape[2]:
            q = u @ u.mT
            u = (a * eye + q @ (b * eye + c * q)) @ u
        else:
            q = u.mT @ u
            u = u @ (a * eye + q @ (b * eye + c * q))
    return u


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "scan_step":
        slots = s["slots"].long()
        a = 1 / (1 + torch.exp(-s["gate"].double()))
        state = s["state"].double()
        state[slots] = a * state[slots] + (1 - a) * s["x"].double()
        return dict(y=state[slots], state=state)
    if kind == "scan_sharded":
        zero = torch.zeros(case["channels"], dtype=torch.float64, device="cuda")
        h, dg, dx, back = _exact_scan(s["gate"], s["x"], zero, s["dy"], zero)
        at = torch.tensor([0] + s["lengths"]).cumsum(0)[:-1].cuda()
        return dict(y=h[1:], dgate=dg, dx=dx, h0=h[at], dlast=torch.cat([back[at[1:]], zero[None]]))
    if kind.startswith("scan"):
        out = dict(y=[], last=[], dgate=[], dx=[], dh0=[])
        at = 0
        for i, n in enumerate(s["lengths"]):
            h0 = s["h0"][i].double()
            part = slice(at, at + n)
            at += n
            if n == 0:
                out["last"].append(h0)
                if kind == "scan_train":
                    out["dh0"].append(s["dlast"][i].double())
                continue
            train = kind == "scan_train"
            h, dg, dx, back = _exact_scan(s["gate"][part], s["x"][part], h0, s["dy"][part] if train else None,
                                          s["dlast"][i] if train else None)
            out["y"].append(h[1:])
            out["last"].append(h[-1])
            if train:
                out["dgate"].append(dg)
                out["dx"].append(dx)
                out["dh0"].append(back[0])
        return {name: (torch.stack if name in ("last", "dh0") else torch.cat)(v) for name, v in out.items() if v}
    if kind == "ortho":
        return _exact_ortho(s["update"])
    if kind == "muon":
        g = s["update"].double()
        m = s["momentum"].double() * MOMENTUM + g
        step = _exact_ortho(m * MOMENTUM + g)
        return dict(weight=s["weight"].double() * (1 - LR * DECAY) - step * (LR * _scale(case)), momentum=m)
    # router: the choice is of whole numbers, given for completeness of the layout
    k, e, tokens = case["k"], case["experts"], s["tokens"]
    keep = s["mask"].bool()
    l = s["logits"].double()[keep]
    shifted = torch.exp(l - l.max(1, keepdim=True).values)
    p = shifted / shifted.sum(1, keepdim=True)
    lse = l.max(1).values + torch.log(shifted.sum(1))
    # stable order, so that of equal logits the lowest index comes first
    order = torch.argsort(-l, dim=1, stable=True)[:, :k]
    w = torch.take_along_dim(p, order, 1)
    norm = w.sum(1, keepdim=True) if case["renormalize"] else torch.ones_like(w[:, :1])
    weights = torch.zeros(len(keep), k, dtype=torch.float64, device="cuda")
    weights[keep] = w / norm
    rank = torch.repeat_interleave(torch.arange(len(tokens)), torch.tensor(tokens)).cuda()[keep]
    sums = torch.zeros(len(tokens), e + 1, dtype=torch.float64, device="cuda")
    sums.index_add_(0, rank, torch.cat([p, lse.square()[:, None]], 1))
    out = dict(indices=None, weights=weights, counts=None, sums=sums)
    if kind == "router_forward":
        return out
    number = max(1, int(keep.sum()))
    f = torch.bincount(order.reshape(-1), minlength=e).double() / (number * k)
    out["loss"] = ALPHA * e / number * (sums[:, :e] @ f) + BETA / number * sums[:, e]
    # gradient by the chain rule through p: dL/dl = p (dL/dp - <p, dL/dp>), then the term of the logits' size
    dw = s["dweights"].double()[keep]
    dp = (ALPHA * e / number * f).expand_as(p).clone()
    dp.scatter_add_(1, order, dw / norm - ((dw * w).sum(1, keepdim=True) / norm ** 2 if case["renormalize"] else 0))
    d = p * (dp - (p * dp).sum(1, keepdim=True)) + 2 * BETA / number * lse[:, None] * p
    out["dlogits"] = torch.zeros(len(keep), e, dtype=torch.float64, device="cuda")
    out["dlogits"][keep] = d
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------


def work(case):
    kind, es = case["kind"], SIZE[case["dtype"]]
    if kind == "scan_step":
        n = case["rows"] * case["channels"]
        # states that no row touches are the caller's own and stay where they are
        return dict(bytes=n * (3 * es + 8) + 4 * case["rows"], flops=8 * n)
    if kind.startswith("scan"):
        lengths, d = _ints(case["lengths"]), case["channels"]
        n, s = sum(lengths) * d, len(lengths) * d
        if kind == "scan_forward":
            return dict(bytes=3 * n * es + 8 * s, flops=8 * n)
        return dict(bytes=6 * n * es + 16 * s, flops=24 * n)
    if kind in ("ortho", "muon"):
        c, m, n = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # the Gram matrix and the polynomial of it are symmetric: half of each suffices
        flops = 5 * c * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
        each = (2 * es) if kind == "ortho" else (3 * es + 8)
        return dict(bytes=c * m * n * each, flops=flops)
    tokens, e, k = _ints(case["tokens"]), case["experts"], case["k"]
    rows, ranks = sum(tokens), len(tokens)
    forward = rows * (e * es + 1 + 8 * k) + ranks * (e + 1) * 8
    if kind == "router_forward":
        return dict(bytes=forward, flops=6 * rows * e)
    return dict(bytes=forward + rows * (e * es + 4 * k) + 4 * ranks, flops=16 * rows * e)
