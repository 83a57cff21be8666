"""Measured cases of the operators around the recurrence, the router and the orthogonalised update of a divided
training step.

Three operators, each of which has one allgather in its middle when the step is divided over the ranks of a
communicator: linear attention with a decay for each head (a sequence divided by time: the ranks exchange the
states that their slices leave), the root-mean-square norm with the residual's addition in front of it and an
8-bit result behind it (rows divided over the ranks: what is exchanged is the 8-bit rows with their scales), and
the norm of all gradients with their clipping (tensors divided over the ranks: the ranks exchange their sums).

`run` computes them in elementary torch operations where `own` is false, in 32 bits (the sums of the gradients'
squares in 64) with one rounding at the end, and through the library where it is true.  `exact` has the same
results in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
CHUNK = 128
LARGEST_E4M3 = 448.0


def listed():
    return [
        # one token for each of 32 running sequences, their states in a table of more slots: serving
        dict(name="attention_step_32", kind="attn_step", rows=32, slots=40, heads=16, keys=128, values=128, dtype="bf16"),
        # one prompt of an odd length on few heads: prefill
        dict(name="attention_prompt_4097", kind="attn_forward", lengths="4097", heads=8, keys=128, values=128,
             dtype="bf16"),
        # packed documents of very different lengths, one of them empty and one a single token, in 32 bits
        dict(name="attention_packed_f32", kind="attn_train", lengths="1,0,777,1501,64,900", heads=8, keys=64, values=64,
             dtype="f32"),
        # an ordinary training batch: 8 sequences, forward and backward
        dict(name="attention_batch_train", kind="attn_train", lengths=",".join(["4096"] * 8), heads=16, keys=128,
             values=128, dtype="bf16"),
        # one long sequence divided over 8 ranks by time, keys narrower than values: states, their allgather, forward
        # and backward
        dict(name="attention_sharded_long", kind="attn_sharded", lengths=",".join(["4096"] * 8), heads=16, keys=64,
             values=128, dtype="f16"),
        # the rows of one step of serving, with 8-bit rows for the products behind
        dict(name="norm_serving_8bit", kind="norm_forward", rows=48, width=4096, block=128, dtype="bf16", weight="bf16"),
        # a prompt of odd width, one scale a row
        dict(name="norm_prompt_8bit", kind="norm_forward", rows=16384, width=5000, block=0, dtype="f16", weight="f16"),
        # a training batch at the width of the step's matrices, both directions
        dict(name="norm_batch_train", kind="norm_train", rows=32768, width=4096, block=0, dtype="bf16", weight="f32"),
        # heads of their own, narrow and odd, in 32 bits, both directions
        dict(name="norm_heads_train", kind="norm_train", rows=200000, width=100, block=0, dtype="f32", weight="f32"),
        # the gradients of a small model on one rank: latency
        dict(name="clip_small", kind="clip", tensors=24, largest=60000, ranks=1, dtype="f32", size="large"),
        # the gradients of a model with their tensors divided over 8 ranks: two types, biases to embeddings
        dict(name="clip_divided", kind="clip", tensors=200, largest=16000000, ranks=8, dtype="bf16", size="large"),
        # gradients that are small enough to stay as they are
        dict(name="clip_kept", kind="clip", tensors=60, largest=4000000, ranks=2, dtype="bf16", size="small"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn_step", "attn_forward", "attn_train", "attn_sharded", "norm_forward", "norm_train", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind.startswith("attn"):
        sizes = [16, 32, 64, 64, 80, 96, 100, 128, 128]
        keys = rng.choice(sizes)
        values = keys if rng.random() < 0.6 else rng.choice(sizes)
        if kind == "attn_step":
            rows = _log(rng, 1, 256)
            return dict(kind=kind, rows=rows, slots=rows + rng.randrange(0, 32), heads=_log(rng, 1, 32), keys=keys,
                        values=values, dtype=dtype)
        heads = _log(rng, 1, 32)
        n = rng.randrange(2, 9) if kind == "attn_sharded" else _log(rng, 1, 16)
        most = max(64, min(32768, (1 << 25) // (heads * 128)) // n)
        return dict(kind=kind, lengths=",".join(str(_log(rng, 1, most)) for _ in range(n)), heads=heads, keys=keys,
                    values=values, dtype=dtype)
    if kind.startswith("norm"):
        width = _log(rng, 32, 16384)
        rows = _log(rng, 1, max(2, (1 << 26) // width))
        return dict(kind=kind, rows=rows, width=width, block=rng.choice([0, 32, 64, 128]) if kind == "norm_forward" else 0,
                    dtype=dtype, weight=rng.choice([dtype, "f32"]))
    return dict(kind=kind, tensors=_log(rng, 1, 300), largest=_log(rng, 100, 8000000), ranks=rng.randrange(1, 9),
                dtype=dtype, size=rng.choice(["large", "large", "small"]))


def _ints(text):
    return [int(v) for v in text.split(",")]


# ---- inputs ----------------------------------------------------------------------------------------------


def _clip_lengths(case):
    """Lengths of the tensors, the same for every seed: matrices, and small ones (biases, norms) beside them."""
    n, most = case["tensors"], case["largest"]
    lengths = [most]
    for i in range(1, n):
        part = most // (3 + i * 7 % 29)
        lengths.append(max(1, part if i % 3 else int(math.sqrt(part)) + i % 5))
    return lengths


def _clip_tensors(case):
    """(type, rank, first element, length) of every tensor; those of one type lie in one buffer, each from a multiple
    of 64 elements on.  Every fifth is held in 32 bits."""
    at, tensors = {}, []
    for i, n in enumerate(_clip_lengths(case)):
        t = "f32" if i % 5 == 4 else case["dtype"]
        start = at.get(t, 0)
        tensors.append((t, i % case["ranks"], start, n))
        at[t] = start + (n + 63) // 64 * 64
    return tensors, at


def _inputs(case, seed):
    """The case's inputs on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["dtype"]]
    kind = case["kind"]

    def normal(*shape, mean=0.0, std=1.0, dtype=t):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean).to(dtype)

    s = dict(case=case, dtype=t)
    if kind.startswith("attn"):
        h, dk, dv = case["heads"], case["keys"], case["values"]
        lengths = _ints(case["lengths"]) if kind != "attn_step" else [1] * case["rows"]
        rows, n = sum(lengths), len(lengths)
        # one projection makes all three, so that their rows lie far apart
        qkv = normal(rows, h * (2 * dk + dv))
        s["q"], s["k"], s["v"] = (p.unflatten(1, (h, -1)) for p in qkv.split([h * dk, h * dk, h * dv], 1))
        # heads that remember from two tokens to a thousand
        s["log_decay"] = torch.log1p(-torch.exp2(-1 - 9 * torch.arange(h, device="cuda", dtype=torch.float64) / h)).float()
        s["scale"] = dk ** -0.5
        if kind == "attn_step":
            s["state"] = normal(case["slots"], h, dk, dv, std=0.3, dtype=torch.float32)
            s["slots"] = torch.randperm(case["slots"], generator=g, device="cuda")[:rows].to(torch.int32)
            return s
        s["lengths"] = lengths
        if kind != "attn_sharded":
            s["first"] = normal(n, h, dk, dv, std=0.3, dtype=torch.float32)
        if kind != "attn_forward":
            s["do"] = normal(rows, h, dv, std=1e-2)
        if kind == "attn_train":
            s["dlast"] = normal(n, h, dk, dv, std=1e-2, dtype=torch.float32)
    elif kind.startswith("norm"):
        rows, w = case["rows"], case["width"]
        s["x"], s["residual"] = normal(rows, w), normal(rows, w, std=2.0)
        s["weight"] = normal(w, mean=1.0, std=0.1, dtype=DTYPES[case["weight"]])
        if kind == "norm_train":
            s["dy"], s["dsum"] = normal(rows, w, std=1e-2), normal(rows, w, std=1e-2)
    else:
        tensors, sizes = _clip_tensors(case)
        std = 1e-2 if case["size"] == "large" else 1e-6
        s["grads"] = {}
        for name, size in sizes.items():
            s["grads"][name] = torch.zeros(size, dtype=DTYPES[name], device="cuda")
        for name, _, start, n in tensors:
            s["grads"][name][start:start + n] = normal(n, std=std, dtype=DTYPES[name])
        s["tensors"], s["most"] = tensors, 1.0
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2109_08751_b200 as sp

    kind, t = case["kind"], s["dtype"]
    codes = {"f32": sp.F32, "bf16": sp.BF16, "f16": sp.F16}
    code = codes[case["dtype"]]
    s["sp"], s["code"] = sp, code

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def with_workspace(plan):
        s["plan"] = plan
        if plan.workspace_bytes:
            plan.set_workspace(empty(plan.workspace_bytes, dtype=torch.uint8), plan.workspace_bytes)

    if kind.startswith("attn"):
        h, dk, dv = case["heads"], case["keys"], case["values"]
        ld = s["q"].stride(0)
        s["ld"] = dict(q_ld=ld, k_ld=ld, v_ld=ld)
        rows = s["q"].shape[0]
        s["o"] = empty(rows, h, dv, dtype=t)
        if kind == "attn_step":
            s["state_out"] = s["state"].clone()
            return s
        n = len(s["lengths"])
        with_workspace(sp.LinearAttentionPlan(s["lengths"], h, dk, dv, code, scale=s["scale"]))
        s["summary"] = empty(n, h * (1 + dk * dv))
        if kind != "attn_forward":
            s["dq"], s["dk"], s["dv"] = empty(rows, h, dk, dtype=t), empty(rows, h, dk, dtype=t), empty(rows, h, dv, dtype=t)
            s["dsummary"] = empty(n, h * (1 + dk * dv))
        if kind == "attn_sharded":
            s["gather"] = sp.Plan(n, s["summary"].shape[1] * 4)
            s["gathered"] = empty(n, n, s["summary"].shape[1])
            s["first"], s["dlast"] = empty(n, h, dk, dv), empty(n, h, dk, dv)
    elif kind.startswith("norm"):
        rows, w, block = case["rows"], case["width"], case["block"]
        with_workspace(sp.NormPlan(w, code, weight_dtype=codes[case["weight"]], eps=EPS, block=block))
        s["sum"], s["rstd"] = empty(rows, w, dtype=t), empty(rows)
        if kind == "norm_forward":
            s["y8"] = empty(rows, w, dtype=torch.float8_e4m3fn)
            s["scales"] = empty(rows, -(-w // block) if block else 1)
        else:
            s["y"], s["dx"], s["dweight"] = empty(rows, w, dtype=t), empty(rows, w, dtype=t), empty(w)
    else:
        ranks = case["ranks"]
        with_workspace(sp.ClipPlan([n for *_, n in s["tensors"]], [codes[name] for name, *_ in s["tensors"]],
                                   ranks=[r for _, r, *_ in s["tensors"]], n_ranks=ranks))
        s["clipped"] = {name: torch.zeros_like(g) for name, g in s["grads"].items()}
        s["plan"].set_tensors(*([buffers[name][start:start + n] for name, _, start, n in s["tensors"]]
                                for buffers in (s["grads"], s["clipped"])))
        s["sums"], s["norms"] = empty(ranks, dtype=torch.float64), empty(ranks, 2)
        s["gather"], s["gathered"] = sp.Plan(ranks, 8), empty(ranks, ranks, dtype=torch.float64)
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---- through the library ---------------------------------------------------------------------------------


def _run_own(s):
    case, kind, sp = s["case"], s["case"]["kind"], s["sp"]
    plan = s.get("plan")
    stream = torch.cuda.current_stream()
    if kind == "attn_step":
        sp.linear_attention_step(case["rows"], case["heads"], case["keys"], case["values"], s["code"], s["q"], s["k"],
                                 s["v"], s["log_decay"], s["state"], s["state_out"], s["o"], scale=s["scale"],
                                 slots=s["slots"], n_slots=case["slots"], stream=stream, **s["ld"])
        return dict(o=s["o"], state=s["state_out"])
    if kind.startswith("attn"):
        h, dk, dv = case["heads"], case["keys"], case["values"]
        n = len(s["lengths"])
        args = (s["q"], s["k"], s["v"], s["log_decay"])
        if kind == "attn_sharded":
            # every rank's slice from nothing; all ranks learn what each leaves; each works out where it starts
            plan.forward(*args, None, summary=s["summary"], stream=stream, **s["ld"])
            s["gather"].allgather(s["summary"], s["gathered"], stream=stream)
            sp.linear_attention_join(n, h, dk, dv, s["gathered"], s["first"], stream=stream)
            plan.forward(*args, s["o"], first=s["first"], stream=stream, **s["ld"])
            # and the same against time for the gradient
            plan.backward(*args, s["do"], None, None, None, dsummary=s["dsummary"], stream=stream, **s["ld"])
            s["gather"].allgather(s["dsummary"], s["gathered"], stream=stream)
            sp.linear_attention_join(n, h, dk, dv, s["gathered"], s["dlast"], reverse=True, stream=stream)
            plan.backward(*args, s["do"], s["dq"], s["dk"], s["dv"], first=s["first"], dlast=s["dlast"], stream=stream,
                          **s["ld"])
            return dict(o=s["o"], dq=s["dq"], dk=s["dk"], dv=s["dv"], first=s["first"], dlast=s["dlast"])
        plan.forward(*args, s["o"], first=s["first"], summary=s["summary"], stream=stream, **s["ld"])
        out = dict(o=s["o"], last=s["summary"][:, h:].unflatten(1, (h, dk, dv)))
        if kind == "attn_forward":
            return out
        plan.backward(*args, s["do"], s["dq"], s["dk"], s["dv"], first=s["first"], dlast=s["dlast"],
                      dsummary=s["dsummary"], stream=stream, **s["ld"])
        return dict(out, dq=s["dq"], dk=s["dk"], dv=s["dv"], dfirst=s["dsummary"][:, h:].unflatten(1, (h, dk, dv)))
    if kind == "norm_forward":
        plan.forward(case["rows"], s["x"], s["weight"], residual=s["residual"], sum=s["sum"], y8=s["y8"],
                     scales=s["scales"], stream=stream)
        return dict(sum=s["sum"], y8=s["y8"], scales=s["scales"])
    if kind == "norm_train":
        plan.forward(case["rows"], s["x"], s["weight"], residual=s["residual"], sum=s["sum"], y=s["y"], rstd=s["rstd"],
                     stream=stream)
        plan.backward(case["rows"], s["dy"], s["sum"], s["weight"], s["rstd"], s["dx"], s["dweight"], dsum=s["dsum"],
                      stream=stream)
        return dict(sum=s["sum"], y=s["y"], dx=s["dx"], dweight=s["dweight"])
    plan.sums(s["sums"], stream=stream)
    s["gather"].allgather(s["sums"], s["gathered"], stream=stream)
    plan.scale(s["gathered"], case["ranks"], s["most"], s["norms"], eps=EPS, stream=stream)
    return dict(s["clipped"], norm=s["norms"][0, 0])


# ---- plain forms -----------------------------------------------------------------------------------------


def _attend(a, b, c, log_decay, z, first):
    """out_t = sum over s <= t of decay^(t - s) (a_t . b_s) c_s  +  decay^(t + first) a_t z, and the state behind the
    last token, in chunks; a, b [T][heads][keys], c [T][heads][values], z [heads][keys][values]."""
    n, dv = a.shape[0], c.shape[2]
    pad = -n % CHUNK  # in front, so that the last chunk is whole

    def chunks(x):
        x = torch.cat([x.new_zeros(pad, *x.shape[1:]), x]) if pad else x
        return x.unflatten(0, (-1, CHUNK)).permute(2, 0, 1, 3)  # [heads][chunks][CHUNK][size]

    a_, b_, c_ = chunks(a), chunks(b), chunks(c)
    l = log_decay[:, None, None]
    at = torch.arange(CHUNK, device=a.device)
    apart = at[:, None] - at[None]
    near = torch.where(apart >= 0, torch.exp(l * apart.clamp_min(0)), 0.0)[:, None]
    left = torch.exp(l * (CHUNK - 1 - at)[:, None])[:, None]          # what a token's part is worth at the chunk's end
    each = (b_ * left).mT @ c_                                         # [heads][chunks][keys][values]
    m = torch.arange(each.shape[1] + 1, device=a.device)
    gap = m[:, None] - 1 - m[None, :-1]
    carried = torch.where(gap >= 0, torch.exp(l * (CHUNK * gap.clamp_min(0))), 0.0)
    state = (carried @ each.flatten(2)).unflatten(2, each.shape[2:])   # in front of every chunk, and behind the last
    entered = torch.exp(l * (at + 1)[:, None])[:, None]
    out = ((a_ @ b_.mT) * near) @ c_ + (a_ @ state[:, :-1]) * entered
    out = out.permute(1, 2, 0, 3).reshape(-1, a.shape[1], dv)[pad:]
    t = torch.arange(n, device=a.device) + first
    far = torch.exp(log_decay[None] * t[:, None])[:, :, None]
    out = out + far * (a.transpose(0, 1) @ z).transpose(0, 1)
    return out, state[:, -1] + torch.exp(l * (n - 1 + first)) * z


def _plain_attention(s):
    case, t = s["case"], s["dtype"]
    h, dk, dv = case["heads"], case["keys"], case["values"]
    l, scale = s["log_decay"], s["scale"]
    lengths = [sum(s["lengths"])] if case["kind"] == "attn_sharded" else s["lengths"]
    zero = torch.zeros(len(lengths), h, dk, dv, device="cuda")
    first, dlast = s.get("first", zero), s.get("dlast", zero)
    if case["kind"] == "attn_sharded":  # the slices make up one sequence
        first = dlast = zero
    parts = {name: [] for name in ("o", "last", "dq", "dk", "dv", "dfirst")}
    at = 0
    for i, n in enumerate(lengths):
        if n == 0:
            parts["last"].append(first[i])
            parts["dfirst"].append(dlast[i])
            continue
        q, k, v = (s[x][at:at + n].float() for x in "qkv")
        o, last = _attend(q, k, v, l, first[i], 1)
        parts["o"].append((scale * o).to(t))
        parts["last"].append(last)
        if "do" in s:
            do = s["do"][at:at + n].float()
            parts["dq"].append((scale * _attend(do, v, k, l, first[i].mT, 1)[0]).to(t))
            q, k, v, do = (scale * q).flip(0), k.flip(0), v.flip(0), do.flip(0)
            dv_, back = _attend(k, q, do, l, dlast[i], 0)
            parts["dv"].append(dv_.flip(0).to(t))
            parts["dk"].append(_attend(v, do, q, l, dlast[i].mT, 0)[0].flip(0).to(t))
            parts["dfirst"].append(torch.exp(l)[:, None, None] * back)
        at += n
    if case["kind"] == "attn_forward":
        return dict(o=torch.cat(parts["o"]), last=torch.stack(parts["last"]))
    rows = {name: torch.cat(parts[name]) for name in ("o", "dq", "dk", "dv")}
    if case["kind"] == "attn_train":
        return dict(rows, last=torch.stack(parts["last"]), dfirst=torch.stack(parts["dfirst"]))
    # what enters each slice, from the slices before and behind it
    each, back, at = [], [], 0
    nothing = zero[0]
    for n in s["lengths"]:
        q, k, v, do = (s[x][at:at + n].float() for x in ("q", "k", "v", "do"))
        left = torch.exp(l[None] * torch.arange(n - 1, -1, -1, device="cuda")[:, None])[:, :, None]
        each.append(torch.einsum("thk,thv->hkv", k * left, v))
        left = torch.exp(l[None] * torch.arange(1, n + 1, device="cuda")[:, None])[:, :, None]
        back.append(torch.einsum("thk,thv->hkv", q * left * scale, do))
        at += n
    firsts, lasts = [nothing], [nothing]
    for n, e in zip(s["lengths"][:-1], each):
        firsts.append(torch.exp(l * n)[:, None, None] * firsts[-1] + e)
    for n, e in zip(s["lengths"][:0:-1], back[:0:-1]):
        lasts.append(torch.exp(l * n)[:, None, None] * lasts[-1] + e)
    return dict(rows, first=torch.stack(firsts), dlast=torch.stack(lasts[::-1]))


def _blocks(y, block):
    """[rows][width] as [rows][scales][columns of a scale], padded with zeros."""
    if not block:
        return y[:, None]
    pad = -y.shape[1] % block
    return torch.nn.functional.pad(y, (0, pad)).unflatten(1, (-1, block))


def _run_plain(s):
    case, kind, t = s["case"], s["case"]["kind"], s["dtype"]
    if kind == "attn_step":
        slots = s["slots"].long()
        q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
        now = torch.exp(s["log_decay"])[:, None, None] * s["state"][slots] + k[..., None] * v[:, :, None]
        state = s["state"].clone()
        state[slots] = now
        return dict(o=(s["scale"] * (q[:, :, None] @ now)[:, :, 0]).to(t), state=state)
    if kind.startswith("attn"):
        return _plain_attention(s)
    if kind.startswith("norm"):
        # the norm is that of the sum as it is kept
        total = (s["x"].float() + s["residual"].float()).to(t)
        r, w = total.float(), s["weight"].float()
        rstd = torch.rsqrt(r.square().mean(1, keepdim=True) + EPS)
        y = r * rstd * w
        if kind == "norm_forward":
            b = _blocks(y, case["block"])
            scales = b.abs().amax(2).clamp_min(1e-30) / LARGEST_E4M3
            y8 = (b / scales[:, :, None]).flatten(1)[:, :case["width"]].to(torch.float8_e4m3fn)
            return dict(sum=total, y8=y8, scales=scales)
        dy, x = s["dy"].float(), r * rstd
        g = dy * w
        dx = rstd * (g - x * (g * x).mean(1, keepdim=True)) + s["dsum"].float()
        return dict(sum=total, y=y.to(t), dx=dx.to(t), dweight=(dy * x).sum(0))
    sums = [s["grads"][name][start:start + n].double().square().sum() for name, _, start, n in s["tensors"]]
    norm = torch.stack(sums).sum().sqrt().float()
    factor = (s["most"] / (norm + EPS)).clamp_max(1.0)
    return dict({name: (g.float() * factor).to(g.dtype) for name, g in s["grads"].items()}, norm=norm)


# ---- 64 bits ---------------------------------------------------------------------------------------------


def _exact_sequence(q, k, v, l, scale, first, do=None, dlast=None):
    """One sequence token by token, the state in hand; [rows][heads][size] each."""
    decay = torch.exp(l.double())[:, None, None]
    q, k, v = (x.double().contiguous() for x in (q, k, v))
    state = first.double().clone()
    o, dq, dk, dv = (torch.empty_like(x) for x in (v, q, k, v))
    if do is not None:
        do = do.double().contiguous()
    for t in range(q.shape[0]):
        torch.baddbmm(decay * state, k[t][:, :, None], v[t][:, None], out=state)
        torch.bmm(q[t][:, None], state, out=o[t][:, None])
        if do is not None:
            torch.bmm(state, do[t][:, :, None], out=dq[t][:, :, None])
    if do is None:
        return o * scale, state, None, None, None, None
    back = dlast.double().clone()
    qs = q * scale
    for t in range(q.shape[0] - 1, -1, -1):
        torch.baddbmm(back, qs[t][:, :, None], do[t][:, None], out=back)  # the gradient of the state behind token t
        torch.bmm(back, v[t][:, :, None], out=dk[t][:, :, None])
        torch.bmm(k[t][:, None], back, out=dv[t][:, None])
        back.mul_(decay)
    return o * scale, state, dq * scale, dk, dv, back


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "attn_step":
        slots = s["slots"].long()
        state = s["state"].double()
        new = state[slots] * torch.exp(s["log_decay"].double()).view(1, -1, 1, 1)
        new += torch.einsum("rhk,rhv->rhkv", s["k"].double(), s["v"].double())
        state[slots] = new
        return dict(o=torch.einsum("rhk,rhkv->rhv", s["q"].double() * s["scale"], new), state=state)
    if kind.startswith("attn"):
        h, dk, dv = case["heads"], case["keys"], case["values"]
        train, sharded = kind != "attn_forward", kind == "attn_sharded"
        if sharded:
            # one sequence in slices: forward through all of them, then back through all of them
            ends = torch.tensor([0] + s["lengths"]).cumsum(0).tolist()
            decay = torch.exp(s["log_decay"].double())[:, None, None]
            q, k, v, do = (s[x].double() for x in ("q", "k", "v", "do"))
            states, backs = [torch.zeros(h, dk, dv, dtype=torch.float64, device="cuda")], []
            backs.append(states[0])
            parts = []
            for i in range(len(s["lengths"])):
                part = slice(ends[i], ends[i + 1])
                parts.append(_exact_sequence(q[part], k[part], v[part], s["log_decay"], s["scale"], states[-1])[0])
                left = decay[:, 0, 0] ** torch.arange(part.stop - part.start - 1, -1, -1, device="cuda")[:, None]
                now = torch.einsum("thk,th,thv->hkv", k[part], left, v[part])
                states.append(decay ** (part.stop - part.start) * states[-1] + now)
            for i in range(len(s["lengths"]) - 1, 0, -1):
                part = slice(ends[i], ends[i + 1])
                left = decay[:, 0, 0] ** torch.arange(1, part.stop - part.start + 1, device="cuda")[:, None]
                now = torch.einsum("thk,th,thv->hkv", q[part] * s["scale"], left, do[part])
                backs.append(decay ** (part.stop - part.start) * backs[-1] + now)
            _, _, dq, dk_, dv_, _ = _exact_sequence(q, k, v, s["log_decay"], s["scale"], states[0], do, backs[0])
            return dict(o=torch.cat(parts), dq=dq, dk=dk_, dv=dv_, first=torch.stack(states[:-1]),
                        dlast=torch.stack(backs[::-1]))
        names = ("o", "last", "dq", "dk", "dv", "dfirst") if train else ("o", "last")
        out = {name: [] for name in names}
        n = s["lengths"]
        if len(set(n)) == 1:  # sequences of one length side by side
            def beside(x):
                return x.unflatten(0, (len(n), n[0])).transpose(0, 1).flatten(1, 2)

            def apart(x):
                return x.unflatten(1, (len(n), h)).transpose(0, 1).flatten(0, 1)

            got = _exact_sequence(*(beside(s[x]) for x in "qkv"), s["log_decay"].repeat(len(n)), s["scale"],
                                  s["first"].flatten(0, 1), beside(s["do"]) if train else None,
                                  s["dlast"].flatten(0, 1) if train else None)
            return {name: x.unflatten(0, (len(n), h)) if name in ("last", "dfirst") else apart(x)
                    for name, x in zip(("o", "last", "dq", "dk", "dv", "dfirst"), got) if name in names}
        at = 0
        for i, m in enumerate(n):
            part = slice(at, at + m)
            at += m
            got = _exact_sequence(*(s[x][part] for x in "qkv"), s["log_decay"], s["scale"], s["first"][i],
                                  s["do"][part] if train else None, s["dlast"][i] if train else None)
            for name, x in zip(("o", "last", "dq", "dk", "dv", "dfirst"), got):
                if name in names:
                    out[name].append(x)
        return {name: (torch.stack if name in ("last", "dfirst") else torch.cat)(x) for name, x in out.items()}
    if kind.startswith("norm"):
        total = s["x"].double() + s["residual"].double()
        kept = total.to(s["dtype"]).double()
        w = s["weight"].double()
        length = torch.sqrt((kept * kept).sum(1, keepdim=True) / case["width"] + EPS)
        unit = kept / length
        if kind == "norm_forward":
            y, block = unit * w, case["block"] or case["width"]
            scales = torch.stack([p.abs().max(1).values for p in y.split(block, 1)], 1) / LARGEST_E4M3
            each = scales.repeat_interleave(block, 1)[:, :case["width"]]
            return dict(sum=total, y8=y / each, scales=scales)
        dy = s["dy"].double()
        du = dy * w
        dx = du / length - kept * (du * kept).sum(1, keepdim=True) / (case["width"] * length ** 3) + s["dsum"].double()
        return dict(sum=total, y=unit * w, dx=dx, dweight=torch.einsum("rc,rc->c", dy, unit))
    norm = torch.sqrt(sum((g.double() ** 2).sum() for g in s["grads"].values()))
    factor = min(1.0, s["most"] / (float(norm) + EPS))
    return dict({name: g.double() * factor for name, g in s["grads"].items()}, norm=norm)


# ---- what a pass cannot do without -----------------------------------------------------------------------


def work(case):
    kind, es = case["kind"], SIZE[case["dtype"]]
    if kind.startswith("attn"):
        h, dk, dv = case["heads"], case["keys"], case["values"]
        if kind == "attn_step":
            rows = case["rows"]
            # states that no row touches are the caller's own and stay where they are
            return dict(bytes=rows * h * (2 * (dk + dv) * es + 8 * dk * dv) + 4 * rows, flops=5 * rows * h * dk * dv)
        lengths = _ints(case["lengths"])
        n, state = sum(lengths) * h, 4 * len(lengths) * h * dk * dv
        # a token updates its state and reads it: 4 keys x values; backward the state once more with one product, the
        # gradient's with two
        if kind == "attn_forward":
            return dict(bytes=n * 2 * (dk + dv) * es + 2 * state, flops=4 * n * dk * dv)
        return dict(bytes=n * (4 * dk + 4 * dv) * es + (2 if kind == "attn_sharded" else 4) * state,
                    flops=14 * n * dk * dv)
    if kind.startswith("norm"):
        n, w = case["rows"] * case["width"], case["width"]
        if kind == "norm_forward":
            scales = case["rows"] * (-(-w // case["block"]) if case["block"] else 1)
            return dict(bytes=n * (3 * es + 1) + 4 * scales + w * SIZE[case["weight"]], flops=8 * n)
        return dict(bytes=n * 7 * es + w * (SIZE[case["weight"]] + 4), flops=18 * n)
    total = sum(n * SIZE[t] for t, _, _, n in _clip_tensors(case)[0])
    return dict(bytes=2 * total + 4, flops=3 * sum(_clip_lengths(case)))
