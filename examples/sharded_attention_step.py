"""One training step of a linear-attention layer whose sequence, rows and gradients are divided over P ranks.

    r = x + residual --norm--> u --W_in--> [q | k | v] --linear attention--> o --W_out--> out

The P ranks are virtual ranks of one GPU, as everywhere in this library; every exchange between them is an allgather of
the library:

  norm        rank r holds a slice of the rows.  Where the rows are wanted everywhere, they are gathered in 8 bits with
              their scales (`share`).
  attention   rank r holds a slice of the sequence.  What each slice leaves of a state is gathered and folded into each
              rank's first state; in the backward pass the same happens against time.
  gradients   rank r owns a block of rows of each.  The ranks' sums of squares are gathered, all gradients are clipped by
              their common norm, and then the rows are gathered for the orthogonalised update.

    python examples/sharded_attention_step.py --ranks 8 --tokens 16384 --steps 5
"""
from __future__ import annotations

import argparse
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2109_08751_b200 as sp  # noqa: E402

CODES = {torch.float32: sp.F32, torch.bfloat16: sp.BF16, torch.float16: sp.F16}


def _planned(plan):
    """The plan with a workspace of its own."""
    ws = torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    plan.set_workspace(ws, ws.numel())
    return plan


class ShardedAttentionStep:
    """Plans, buffers and weights of the step; `gradients` goes forward and back, `update` clips and updates."""

    def __init__(self, tokens_per_rank, width: int, heads: int, size: int, dtype=torch.bfloat16, most: float = 1.0,
                 lr: float = 0.02, block: int = 128, seed: int = 0):
        P, T, code, inner = len(tokens_per_rank), sum(tokens_per_rank), CODES[dtype], heads * size
        if width % P or inner % P:
            raise ValueError("every rank owns the same number of rows of a matrix")
        self.tokens, self.P, self.T, self.dtype, self.code = list(tokens_per_rank), P, T, dtype, code
        self.width, self.heads, self.size, self.inner, self.most, self.lr = width, heads, size, inner, most, lr
        g = torch.Generator(device="cuda").manual_seed(seed)

        def new(*shape, dt=torch.float32):
            return torch.empty(*shape, dtype=dt, device="cuda")

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") / math.sqrt(rows)).to(dtype)

        self.weights = {"in": weight(width, 3 * inner), "out": weight(inner, width)}
        self.scale = torch.ones(width, device="cuda")  # the norm's weight
        self.log_decay = torch.log1p(-torch.exp2(-1 - 8 * torch.arange(heads, device="cuda") / heads))
        self.momentum = {n: torch.zeros_like(w, dtype=torch.float32) for n, w in self.weights.items()}
        self.norm = _planned(sp.NormPlan(width, code, weight_dtype=sp.F32, block=block))
        self.attention = _planned(sp.LinearAttentionPlan(self.tokens, heads, size, size, code))
        self.ortho = {n: _planned(sp.OrthoPlan(1, *w.shape, code)) for n, w in self.weights.items()}
        # gradients: rank r's rows of each matrix; the norm's weight is rank 0's
        self.grads = {n: torch.zeros_like(w) for n, w in self.weights.items()}
        self.dscale = torch.zeros(width, device="cuda")
        owned = [(r, rows) for n in self.grads for r, rows in enumerate(self.grads[n].chunk(P))] + [(0, self.dscale)]
        self.clip = _planned(sp.ClipPlan([t.numel() for _, t in owned], [CODES[t.dtype] for _, t in owned],
                                         ranks=[r for r, _ in owned], n_ranks=P))
        self.clip.set_tensors([t for _, t in owned], [t for _, t in owned])
        # what the ranks gather: states, sums, rows of a gradient
        block_size = heads * (1 + size * size)
        self.summary, self.summaries = new(P, block_size), new(P, P, block_size)
        self.first, self.last = new(P, heads, size, size), new(P, heads, size, size)
        self.gather_states = sp.Plan(P, block_size * 4)
        self.sums, self.all_sums, self.norms = new(P, dt=torch.float64), new(P, P, dt=torch.float64), new(P, 2)
        self.gather_sums = sp.Plan(P, 8)
        self.gather_rows = {n: sp.Plan(P, w.numel() // P * w.element_size()) for n, w in self.weights.items()}
        self.r, self.u, self.o, self.do = (new(T, w, dt=dtype) for w in (width, width, inner, inner))
        self.rstd, self.dx, self.dqkv = new(T), new(T, width, dt=dtype), new(T, 3 * inner, dt=dtype)

    def _parts(self, x):
        return (x[:, i * self.inner:(i + 1) * self.inner] for i in range(3))

    def forward(self, x, residual):
        """out [T][width]; the sum of x and residual stays in `r`."""
        stream, ld = torch.cuda.current_stream(), 3 * self.inner
        self.norm.forward(self.T, x, self.scale, residual=residual, sum=self.r, y=self.u, rstd=self.rstd, stream=stream)
        self.qkv = self.u @ self.weights["in"]
        q, k, v = self._parts(self.qkv)
        # what each slice leaves, everybody's, where each slice starts, the outputs
        self.attention.forward(None, k, v, self.log_decay, None, summary=self.summary, k_ld=ld, v_ld=ld, stream=stream)
        self.gather_states.allgather(self.summary, self.summaries, stream=stream)
        sp.linear_attention_join(self.P, self.heads, self.size, self.size, self.summaries, self.first, stream=stream)
        self.attention.forward(q, k, v, self.log_decay, self.o, first=self.first, q_ld=ld, k_ld=ld, v_ld=ld, stream=stream)
        return self.o @ self.weights["out"]

    def gradients(self, x, residual, dout, dr=None):
        """Forward and back; dr: gradient that reaches r on other ways.  Returns out and the gradient of x (and residual);
        those of the weights are in `grads` and `dscale`."""
        out = self.forward(x, residual)
        stream, ld = torch.cuda.current_stream(), 3 * self.inner
        torch.matmul(self.o.T, dout, out=self.grads["out"])
        torch.matmul(dout, self.weights["out"].T, out=self.do)
        q, k, v = self._parts(self.qkv)
        dq, dk, dv = self._parts(self.dqkv)
        self.attention.backward(q, None, None, self.log_decay, self.do, None, None, None, dsummary=self.summary, q_ld=ld,
                                stream=stream)
        self.gather_states.allgather(self.summary, self.summaries, stream=stream)
        sp.linear_attention_join(self.P, self.heads, self.size, self.size, self.summaries, self.last, reverse=True,
                                 stream=stream)
        self.attention.backward(q, k, v, self.log_decay, self.do, dq, dk, dv, first=self.first, dlast=self.last, q_ld=ld,
                                k_ld=ld, v_ld=ld, dq_ld=ld, dk_ld=ld, dv_ld=ld, stream=stream)
        torch.matmul(self.u.T, self.dqkv, out=self.grads["in"])
        du = self.dqkv @ self.weights["in"].T
        self.norm.backward(self.T, du, self.r, self.scale, self.rstd, self.dx, self.dscale, dsum=dr, stream=stream)
        return out, self.dx

    def update(self):
        """Clips all gradients by their common norm and updates the weights; returns the norm."""
        stream = torch.cuda.current_stream()
        self.clip.sums(self.sums, stream=stream)
        self.gather_sums.allgather(self.sums, self.all_sums, stream=stream)
        self.clip.scale(self.all_sums, self.P, self.most, self.norms, stream=stream)
        for name, w in self.weights.items():
            full = torch.empty(self.P, *w.shape, dtype=self.dtype, device="cuda")
            self.gather_rows[name].allgather(self.grads[name], full, stream=stream)
            # every rank holds the whole gradient now; on one GPU the first one's copy stands for all
            self.ortho[name].muon_step(full[0], self.momentum[name], self.momentum[name], w, w, weight_dtype=self.code,
                                       lr=self.lr, weight_decay=0.01, scale=0.2 * math.sqrt(max(w.shape)), stream=stream)
        self.scale -= self.lr * self.dscale
        return self.norms[0, 0]

    def share(self, x, rows: int):
        """The norm of x [P * rows][width] on every rank, gathered in 8 bits: [P][P * rows][width] e4m3 and its scales."""
        stream = torch.cuda.current_stream()
        per_row = -(-self.width // 128)
        y8 = torch.empty(self.P * rows, self.width, dtype=torch.float8_e4m3fn, device="cuda")
        scales = torch.empty(self.P * rows, per_row, device="cuda")
        plan = sp.NormPlan(self.width, self.code, weight_dtype=sp.F32, block=128)
        plan.forward(self.P * rows, x, self.scale, y8=y8, scales=scales, stream=stream)
        all_8 = torch.empty(self.P, *y8.shape, dtype=y8.dtype, device="cuda")
        all_scales = torch.empty(self.P, *scales.shape, device="cuda")
        sp.Plan(self.P, rows * self.width).allgather(y8, all_8, stream=stream)
        sp.Plan(self.P, rows * per_row * 4).allgather(scales, all_scales, stream=stream)
        return all_8, all_scales

    def status(self) -> None:
        """Waits, and raises where a wait inside a kernel gave up."""
        plans = [self.attention, *self.ortho.values(), self.gather_states, self.gather_sums, *self.gather_rows.values()]
        if any(p.status() != sp.OK for p in plans):
            raise RuntimeError("a device-side wait timed out")


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--ranks", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=16384)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--size", type=int, default=128)
    ap.add_argument("--steps", type=int, default=5)
    a = ap.parse_args()
    each = [a.tokens // a.ranks + (r < a.tokens % a.ranks) for r in range(a.ranks)]
    step = ShardedAttentionStep(each, a.width, a.heads, a.size)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, residual = (torch.randn(a.tokens, a.width, generator=g, device="cuda").bfloat16() for _ in range(2))
    dout = (torch.randn(a.tokens, a.width, generator=g, device="cuda") * 1e-6).bfloat16()
    for i in range(a.steps):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        step.gradients(x, residual, dout)
        norm = step.update()
        end.record()
        step.status()
        print(f"step {i}: norm of the gradients {norm.item():.4f}, {start.elapsed_time(end):.2f} ms")


if __name__ == "__main__":
    main()
