"""Linear attention with a decay for each head against the recurrence in 64 bits, token by token.

Tolerances.  With u half a step of the type (bf16 2^-8, fp16 2^-11) and M_t the recurrence over absolute values, o_t
is off by at most u |o_t| for its own rounding and u scale |q_t| M_t for those of the weights (tokens of the chunk) and
of the state (the tokens before), which share the tokens between them.  Everything else is 32-bit arithmetic: 2^-24 for
each of some 400 additions and a factor, below 2^-14 of the same magnitude.  States are 32-bit arithmetic only."""
import random

import pytest
import torch

import paper_2109_08751_b200 as sp

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, sp.BF16, 2.0 ** -8), "f16": (torch.float16, sp.F16, 2.0 ** -11),
         "f32": (torch.float32, sp.F32, 2.0 ** -24)}
SLACK = 2.0 ** -14


def recurrence(q, k, v, decay, scale, first, do=None, dlast=None):
    """One sequence in 64 bits; gradients where do is given."""
    state = first.clone()
    o, dq, dk, dv = (torch.empty_like(x) for x in (v, q, k, v))
    for t in range(q.shape[0]):
        state = decay * state + k[t][:, :, None] * v[t][:, None]
        o[t] = scale * (q[t][:, None] @ state)[:, 0]
        if do is not None:
            dq[t] = scale * (state @ do[t][:, :, None])[:, :, 0]
    if do is None:
        return dict(o=o, last=state)
    back = dlast.clone()
    for t in range(q.shape[0] - 1, -1, -1):
        back = back + scale * q[t][:, :, None] * do[t][:, None]
        dk[t] = (back @ v[t][:, :, None])[:, :, 0]
        dv[t] = (k[t][:, None] @ back)[:, 0]
        back = decay * back
    return dict(o=o, last=state, dq=dq, dk=dk, dv=dv, dfirst=back)


class Case:
    """Inputs, plan and buffers of some sequences; `run` makes the calls."""

    def __init__(self, lengths, heads, kd, vd, name, seed=0, pad=0, decays=None, first=True, scale=None, shift=0):
        self.t, self.code, self.u = TYPES[name]
        self.lengths, self.heads, self.kd, self.vd = lengths, heads, kd, vd
        rows, n = sum(lengths), len(lengths)
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std=1.0, dtype=self.t):
            return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

        def rows_of(size, std=1.0):
            wide = normal(rows, heads * size + pad + shift, std=std)
            return wide[:, shift:shift + heads * size]

        self.q, self.k, self.v, self.do = rows_of(kd), rows_of(kd), rows_of(vd), rows_of(vd, 1e-2)
        if decays is None:
            decays = [1 - 2.0 ** -(1 + 9 * h / heads) for h in range(heads)]
        self.log_decay = torch.tensor(decays, dtype=torch.float64, device="cuda").log().float()
        self.scale = kd ** -0.5 if scale is None else scale
        self.first = normal(n, heads, kd, vd, std=0.3, dtype=torch.float32) if first else None
        self.dlast = normal(n, heads, kd, vd, std=1e-2, dtype=torch.float32) if first else None
        self.plan = sp.LinearAttentionPlan(lengths, heads, kd, vd, self.code, scale=self.scale)
        self.work = torch.empty(self.plan.workspace_bytes, dtype=torch.uint8, device="cuda")
        self.plan.set_workspace(self.work, self.work.numel())
        self.out = {}
        for name_, size in dict(o=vd, dq=kd, dk=kd, dv=vd).items():
            wide = torch.full((rows + 2, heads * size + pad + shift), 7.0, dtype=self.t, device="cuda")
            self.out[name_] = wide
        self.pad, self.shift = pad, shift
        self.summary = torch.full((n, heads * (1 + kd * vd)), 7.0, device="cuda")
        self.dsummary = torch.full_like(self.summary, 7.0)

    def inner(self, name):
        w = self.out[name]
        size = self.vd if name in ("o", "dv") else self.kd
        return w[:sum(self.lengths), self.shift:self.shift + self.heads * size]

    def run(self, backward=True, stream=None):
        ld = lambda x: x.stride(0) if x.shape[0] else x.shape[1]  # noqa: E731
        at = dict(q_ld=ld(self.q), k_ld=ld(self.k), v_ld=ld(self.v), stream=stream)
        self.plan.forward(self.q, self.k, self.v, self.log_decay, self.inner("o"), first=self.first, summary=self.summary,
                          o_ld=self.out["o"].stride(0), **at)
        if backward:
            self.plan.backward(self.q, self.k, self.v, self.log_decay, self.do, self.inner("dq"), self.inner("dk"),
                               self.inner("dv"), first=self.first, dlast=self.dlast, dsummary=self.dsummary,
                               do_ld=ld(self.do), dq_ld=self.out["dq"].stride(0), dk_ld=self.out["dk"].stride(0),
                               dv_ld=self.out["dv"].stride(0), **at)

    def reference(self, backward=True):
        """Values and magnitudes of everything, sequence by sequence."""
        decay = self.log_decay.double().exp()[:, None, None]
        at, all_ = 0, []
        for i, n in enumerate(self.lengths):
            part = slice(at, at + n)
            at += n
            zero = torch.zeros(self.heads, self.kd, self.vd, dtype=torch.float64, device="cuda")
            x = [a[part].double().unflatten(1, (self.heads, -1)) for a in (self.q, self.k, self.v)]
            f = zero if self.first is None else self.first[i].double()
            d = self.do[part].double().unflatten(1, (self.heads, -1)) if backward else None
            e = zero if self.dlast is None else self.dlast[i].double()
            value = recurrence(*x, decay, self.scale, f, d, e)
            size = recurrence(*(a.abs() for a in x), decay, abs(self.scale), f.abs(), d.abs() if backward else None, e.abs())
            all_.append((value, size))
        return all_

    def check(self, backward=True):
        torch.cuda.synchronize()
        assert self.plan.status() == sp.OK
        size = self.kd * self.vd
        at = 0
        for i, (value, most) in enumerate(self.reference(backward)):
            n = self.lengths[i]
            for name in ("o", "dq", "dk", "dv") if backward else ("o",):
                got = self.inner(name)[at:at + n].double().unflatten(1, (self.heads, -1)) if n else value[name]
                rounding = self.u if self.code != sp.F32 else 0.0
                tol = (rounding + SLACK) * most[name] + self.u * value[name].abs() + (2.0 ** -25 if self.code == sp.F16 else 0)
                worst = ((got - value[name]).abs() / tol.clamp_min(1e-30)).max().item() if n else 0.0
                assert worst <= 1.0, (name, i, worst)
            for name, summary in (("last", self.summary), ("dfirst", self.dsummary)) if backward else (("last", self.summary),):
                got = summary[i, self.heads:].double().view(self.heads, self.kd, self.vd)
                worst = ((got - value[name]).abs() / (SLACK * most[name]).clamp_min(1e-30)).max().item()
                assert worst <= 1.0, (name, i, worst)
                want = (self.log_decay.double() * n).exp()
                assert torch.allclose(summary[i, :self.heads].double(), want, rtol=1e-5, atol=1e-38)
            at += n
        assert size > 0
        rows = sum(self.lengths)
        for name, w in self.out.items():  # what lies around the results is as it was
            if name == "o" or backward:
                assert (w[rows:] == 7.0).all()
                width = self.heads * (self.vd if name in ("o", "dv") else self.kd)
                assert (w[:, :self.shift] == 7.0).all() and (w[:, self.shift + width:] == 7.0).all()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,heads,kd,vd", [
    ([128], 1, 128, 128), ([1], 1, 64, 64), ([300], 2, 64, 64), ([7, 0, 129, 256, 1], 3, 128, 128), ([500, 130], 2, 64, 128),
    ([500, 130], 2, 128, 64)])
def test_against_the_recurrence(lengths, heads, kd, vd, name):
    c = Case(lengths, heads, kd, vd, name)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kd,vd,pad,shift", [(100, 80, 0, 0), (80, 100, 4, 0), (16, 48, 0, 0), (33, 17, 1, 1), (1, 1, 0, 0),
                                             (128, 96, 2, 0), (64, 64, 8, 8), (64, 128, 4, 4), (96, 32, 0, 2)])
def test_sizes_strides_and_alignments(kd, vd, pad, shift, name):
    c = Case([200, 3, 129], 3, kd, vd, name, pad=pad, shift=shift)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
def test_long_sequences_in_segments(name):
    # few heads: the plan cuts the long sequences, leaves the short ones, and has an empty one
    c = Case([3000, 0, 1, 257], 2, 64, 64, name)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("kd,vd,lengths", [(128, 128, [900, 768, 1100]), (64, 64, [1500, 1024, 700]), (64, 128, [900, 640, 641])])
def test_long_chains_of_chunks(kd, vd, lengths, name):
    # as many heads as fill the GPU: the plan cuts nothing, and every stage of the kernel's ring is used many times
    c = Case(lengths, 64, kd, vd, name, seed=4)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,heads", [([2000, 1500, 0, 130, 1, 900], 20), ([0, 0, 5, 0, 300], 70), ([1111], 31),
                                           ([700, 0, 1000, 129], 40)])
def test_several_segments_a_processor(lengths, heads, name):
    # more segments than processors, some of them empty or with nothing to add: whoever goes on to the next one has to
    # agree with the others on where it is
    c = Case(lengths, heads, 32, 64, name, seed=6)
    c.run()
    c.check()


@pytest.mark.parametrize("seed", range(12))
def test_drawn_shapes(seed):
    r = random.Random(seed)
    name, sizes = r.choice(["bf16", "f16", "f32"]), [16, 32, 64, 64, 80, 100, 128]
    n, heads = r.randrange(1, 12), r.choice([1, 2, 3, 5, 9, 16, 32])
    c = Case([r.choice([0, 1, r.randrange(1, 300), r.randrange(1, 1200)]) for _ in range(n)], heads, r.choice(sizes),
             r.choice(sizes), name, seed=seed)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_many_short_sequences(name):
    c = Case([1 + i % 130 for i in range(60)], 4, 32, 64, name)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("decays", [[0.0, 1.0], [1e-30, 0.5], [1 - 2.0 ** -20, 1e-3]])
def test_decays_from_nothing_to_everything(decays, name):
    c = Case([300, 70], 2, 64, 64, name, decays=decays, seed=2)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_without_first_states(name):
    c = Case([140, 1], 2, 64, 32, name, first=False, scale=-0.7)
    c.run()
    c.check()


@pytest.mark.parametrize("lengths", [[300, 5], [2600]])
@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
def test_summaries_alone(lengths, name):
    c = Case(lengths, 2, 64, 96, name)
    c.run()
    both = c.summary.clone(), c.dsummary.clone()
    c.summary.fill_(3.0)
    c.dsummary.fill_(3.0)
    n = c.q.stride(0)
    c.plan.forward(None, c.k, c.v, c.log_decay, None, first=c.first, summary=c.summary, k_ld=n, v_ld=c.v.stride(0))
    c.plan.backward(c.q, None, None, c.log_decay, c.do, None, None, None, dlast=c.dlast, dsummary=c.dsummary, q_ld=n,
                    do_ld=c.do.stride(0))
    # the same sums, in segments or along the sequence
    assert torch.allclose(both[0], c.summary, rtol=1e-4, atol=1e-4) and torch.allclose(both[1], c.dsummary, rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
def test_divided_by_time(name):
    """Slices of one sequence with an allgather of what each leaves, against the whole sequence."""
    whole = Case([700], 2, 64, 32, name, first=False)
    whole.run()
    lengths = [128, 1, 0, 400, 171]
    P, part = len(lengths), Case(lengths, 2, 64, 32, name, first=False)
    for x in ("q", "k", "v", "do"):
        getattr(part, x).copy_(getattr(whole, x))
    h, size = 2, 64 * 32
    gather, all_ = sp.Plan(P, part.summary.shape[1] * 4), torch.empty(P, *part.summary.shape, device="cuda")
    at = dict(k_ld=part.k.stride(0), v_ld=part.v.stride(0))
    part.first, part.dlast = torch.empty(P, h, 64, 32, device="cuda"), torch.empty(P, h, 64, 32, device="cuda")
    part.plan.forward(None, part.k, part.v, part.log_decay, None, summary=part.summary, **at)
    gather.allgather(part.summary, all_)
    sp.linear_attention_join(P, h, 64, 32, all_, part.first)
    part.plan.backward(part.q, None, None, part.log_decay, part.do, None, None, None, dsummary=part.dsummary,
                       q_ld=part.q.stride(0), do_ld=part.do.stride(0))
    gather.allgather(part.dsummary, all_)
    sp.linear_attention_join(P, h, 64, 32, all_, part.dlast, reverse=True)
    one = torch.empty(2, h, 64, 32, device="cuda")  # a process that is ranks 1 and 2
    sp.linear_attention_join(P, h, 64, 32, all_[1:], one, reverse=True, first_rank=1, n_ranks=2)
    assert torch.equal(one, part.dlast[1:3])
    part.run()
    torch.cuda.synchronize()
    assert part.plan.status() == sp.OK
    for x in ("o", "dq", "dk", "dv"):
        a, b = part.inner(x).float(), whole.inner(x).float()
        assert (a - b).norm() <= 4 * max(whole.u, 1e-5) * b.norm(), x  # each within two roundings of the truth
    assert part.first.numel() == P * h * size


def close(a, b, u):
    """What the tokens of a chunk that holds such a number are: the same sums in another order, so that each is 32-bit
    arithmetic (2^-14 of the sums' magnitude, here of at most 64 times the largest value) and a rounding from the other."""
    return a.isfinite().all() and ((a - b).abs().double() <= 2 * u * b.abs().double() + 2.0 ** -14 * 64 * b.abs().max()).all()


def test_what_is_not_a_number_reaches_no_token_before_it():
    for name in ("bf16", "f16", "f32"):
        for what in (float("nan"), float("inf")):
            for x, column in (("v", 5), ("k", 9)):
                c = Case([290, 140], 2, 64, 64, name, decays=[0.9, 0.99])
                clean = Case([290, 140], 2, 64, 64, name, decays=[0.9, 0.99])
                clean.run()
                getattr(c, x)[150, 64 + column] = what  # token 150 of the first sequence, second head
                c.run()
                torch.cuda.synchronize()
                assert c.plan.status() == sp.OK
                o, want = (z.inner("o").unflatten(1, (2, 64)) for z in (c, clean))
                assert torch.equal(o[:128], want[:128]) and torch.equal(o[290:], want[290:]) and torch.equal(o[:, 0], want[:, 0])
                assert close(o[128:150], want[128:150], c.u)
                if x == "v":  # its column of values alone, to the end of the sequence
                    assert not torch.isfinite(o[150:290, 1, column]).any()
                    rest = [i for i in range(64) if i != column]
                    assert close(o[128:256, 1, rest], want[128:256, 1, rest], c.u)
                    assert torch.equal(o[256:, 1, rest], want[256:, 1, rest])
                else:
                    assert not torch.isfinite(o[150:290, 1]).any()
                # gradients: do at a token reaches the tokens before it
                d = Case([290, 140], 2, 64, 64, name, decays=[0.9, 0.99])
                d.do[150, 64 + column] = what
                d.run()
                torch.cuda.synchronize()
                dv, want = (z.inner("dv").unflatten(1, (2, 64)) for z in (d, clean))
                # against time the chunks are counted from the end: tokens 34 to 161 are one
                assert torch.equal(dv[162:], want[162:]) and torch.equal(dv[:, 0], want[:, 0])
                assert close(dv[151:162], want[151:162], c.u) and not torch.isfinite(dv[:151, 1, column]).any()
                dk, want = (z.inner("dk").unflatten(1, (2, 64)) for z in (d, clean))
                assert torch.equal(dk[162:], want[162:]) and not torch.isfinite(dk[:151, 1]).any()
                assert close(dk[151:162], want[151:162], c.u)


@pytest.mark.parametrize("k_size,v_size,do_size", [(1.0, 1e-4, 1e-5), (60.0, 300.0, 1e-2), (1e-3, 1e-3, 1.0)])
def test_fp16_numbers_far_from_one(k_size, v_size, do_size):
    """Scores, states and gradients that fp16 itself would round away or not hold."""
    c = Case([2000], 1, 64, 64, "f16", decays=[1 - 2.0 ** -11])
    c.k.mul_(k_size)
    c.v.mul_(v_size)
    c.do.mul_(do_size * 100)
    c.run()
    torch.cuda.synchronize()
    (value, _), = c.reference()
    for x in ("o", "dq", "dk", "dv"):
        got, want = c.inner(x).double(), value[x].flatten(1)
        if want.abs().max() > 6e4:
            continue  # the result itself is none of fp16
        floor = 2.0 ** -25 * want.numel() ** 0.5  # the spacing of its smallest numbers
        assert (got - want).norm() <= 2 * c.u * want.norm() + floor, x


def test_gradient_against_differences():
    c = Case([37, 100], 2, 24, 40, "f32", seed=5)
    c.run()
    g = torch.Generator(device="cuda").manual_seed(1)
    weight, wl = c.do.clone(), c.dlast.clone()

    def loss():
        c.run(backward=False)
        last = c.summary[:, c.heads:].reshape(wl.shape)
        return (c.inner("o").double() * weight.double()).sum() + (last.double() * wl.double()).sum()

    grads = {x: c.inner("d" + x).clone() for x in "qkv"}
    grads["first"] = c.dsummary[:, c.heads:].reshape(c.first.shape).clone()
    for x, grad in grads.items():
        t = getattr(c, x)
        kept, way = t.clone(), torch.randn(t.shape, generator=g, device="cuda")
        step = 0.5  # the loss is linear in each of them
        t.copy_(kept + step * way)
        up = loss()
        t.copy_(kept - step * way)
        down = loss()
        t.copy_(kept)
        slope, want = ((up - down) / (2 * step)).item(), (grad.double() * way.double()).sum().item()
        size = (grad.double() * way.double()).abs().sum().item()
        assert abs(slope - want) <= 1e-5 * size, x


def test_same_bits_on_every_run_and_when_replayed():
    for name in ("bf16", "f16", "f32"):
        c = Case([1500, 200], 2, 64, 64, name)
        c.run()
        torch.cuda.synchronize()
        first = {x: w.clone() for x, w in c.out.items()} | dict(s=c.summary.clone(), d=c.dsummary.clone())
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            c.run(stream=stream)
        for _ in range(3):
            for w in c.out.values():
                w.fill_(7.0)
            c.summary.fill_(0.0)
            graph.replay()
            torch.cuda.synchronize()
            for x, w in first.items():
                assert torch.equal(w, c.summary if x == "s" else c.dsummary if x == "d" else c.out[x]), x


def test_two_plans_on_two_streams():
    a, b = Case([900], 4, 64, 64, "bf16"), Case([900], 4, 128, 128, "f16", seed=3)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        a.run(stream=streams[0])
        b.run(stream=streams[1])
    a.check()
    b.check()


def test_waits_give_up():
    c = Case([700], 2, 64, 64, "bf16")
    c.plan.set_wait_test(True, 20_000_000)
    c.run(backward=False)
    assert c.plan.status() == sp.ERR_TIMEOUT
    c.plan.set_wait_test(False)
    c.run()
    c.check()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,heads,kd,vd", [(1, 1, 128, 128), (5, 3, 64, 100), (40, 16, 128, 128), (300, 2, 33, 17), (3, 2, 1, 1)])
def test_single_tokens(rows, heads, kd, vd, name):
    t, code, u = TYPES[name]
    g = torch.Generator(device="cuda").manual_seed(rows)
    slots = rows + 3
    qkv = torch.randn(rows, heads * (2 * kd + vd) + 5, generator=g, device="cuda").to(t)
    q, k, v = qkv[:, :heads * kd], qkv[:, heads * kd:2 * heads * kd], qkv[:, 2 * heads * kd:heads * (2 * kd + vd)]
    state = torch.randn(slots, heads, kd, vd, generator=g, device="cuda")
    log_decay = torch.log1p(-torch.rand(heads, generator=g, device="cuda"))
    names = torch.randperm(slots, generator=g, device="cuda")[:rows].to(torch.int32)
    if rows > 2:
        names[1], names[2] = -1, slots  # rows without a sequence
    at = dict(q_ld=qkv.stride(0), k_ld=qkv.stride(0), v_ld=qkv.stride(0), slots=names, n_slots=slots)
    o, out = torch.full((rows, heads * vd + 2), 7.0, dtype=t, device="cuda"), state.clone()
    sp.linear_attention_step(rows, heads, kd, vd, code, q, k, v, log_decay, state, out, o, o_ld=o.stride(0), **at)
    there = (names >= 0) & (names < slots)
    n = names[there].long()
    x = [y[there].double().unflatten(1, (heads, -1)) for y in (q, k, v)]
    decay = log_decay.double().exp()[:, None, None]
    want = decay * state[n].double() + x[1][..., None] * x[2][:, :, None]
    size = decay * state[n].double().abs() + x[1].abs()[..., None] * x[2].abs()[:, :, None]
    expected = state.double().clone()
    expected[n] = want
    assert ((out.double() - expected).abs()[n] <= 2.0 ** -21 * size).all()
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[n] = False
    assert torch.equal(out[rest], state[rest])
    wo = kd ** -0.5 * torch.einsum("rhk,rhkv->rhv", x[0], want)
    so = kd ** -0.5 * torch.einsum("rhk,rhkv->rhv", x[0].abs(), size)
    got = o[:, :heads * vd].double().unflatten(1, (heads, vd))
    assert ((got[there] - wo).abs() <= u * wo.abs() + 2.0 ** -16 * so + 2.0 ** -25).all()
    assert (got[~there] == 0).all() and (o[:, heads * vd:] == 7.0).all()
    # in place
    again = state.clone()
    sp.linear_attention_step(rows, heads, kd, vd, code, q, k, v, log_decay, again, again, o, o_ld=o.stride(0), **at)
    assert torch.equal(again, out)


def test_single_tokens_follow_a_prompt():
    """The last state of a prompt goes on token by token as the whole sequence does."""
    c = Case([200], 2, 64, 64, "f32", first=False)
    c.run(backward=False)
    whole = c.inner("o").clone()
    p = Case([197], 2, 64, 64, "f32", first=False)
    for x in ("q", "k", "v"):
        getattr(p, x).copy_(getattr(c, x)[:197])
    p.run(backward=False)
    state = p.summary[:, 2:].reshape(1, 2, 64, 64).clone()
    for t in range(197, 200):
        o = torch.empty(1, 128, device="cuda")
        sp.linear_attention_step(1, 2, 64, 64, sp.F32, c.q[t:t + 1], c.k[t:t + 1], c.v[t:t + 1], c.log_decay, state, state, o)
        assert torch.allclose(o, whole[t:t + 1], rtol=1e-4, atol=1e-5)
