"""Linear attention with a decay for each head against the recurrence in 64 bits, token by token.

Tolerances.  With u half a step of the type (bf16 2^-8, fp16 2^-11) and M_t the recurrence over absolute values, o_t
is off by at most u |o_t| for its own rounding and u scale |q_t| M_t for those of the weights (tokens of the chunk) and
of the state (the tokens before), which share the tokens between them.  Everything else is 32-bit arithmetic: 2^-24 for
each of some 400 additions and a factor, below 2^-14 of the same magnitude.  States are 32-bit arithmetic only."""
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
