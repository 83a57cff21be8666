"""One training step of a small model whose sequence, tokens and matrices are divided over P ranks.

    h --W_in--> [gate | x] --gated recurrence--> y --W_router--> logits --> k experts a token

The P ranks are virtual ranks of one GPU, as everywhere in this library; every exchange between them is
an allgather of the library:

  recurrence   rank r holds a slice of the sequence.  The slices' summaries are gathered and folded into
               each rank's first state; in the backward pass the same happens against time.
  router       the ranks' per-expert counts are gathered: the balance loss compares a rank's
               probabilities with the counts of all ranks.
  matrices     rank r owns a block of rows of each gradient.  The rows are gathered, and the update is
               orthogonalised with the momentum in front of it and the weight update behind it.

    python examples/sharded_training_step.py --ranks 8 --tokens 16384 --steps 5
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


class ShardedStep:
    """Plans, buffers and weights of the step; `run` takes one."""

    def __init__(self, tokens_per_rank, width: int, channels: int, experts: int, k: int, dtype=torch.bfloat16,
                 alpha: float = 1e-2, beta: float = 1e-3, lr: float = 0.02, seed: int = 0):
        P, T, code = len(tokens_per_rank), sum(tokens_per_rank), CODES[dtype]
        if width % P or channels % P:
            raise ValueError("every rank owns the same number of rows of a matrix")
        self.tokens, self.P, self.T, self.dtype, self.code = list(tokens_per_rank), P, T, dtype, code
        self.channels, self.experts, self.k, self.alpha, self.beta, self.lr = channels, experts, k, alpha, beta, lr
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") / math.sqrt(rows)).to(dtype)

        self.weights = {"in": weight(width, 2 * channels), "router": weight(channels, experts)}
        self.momentum = {n: torch.zeros_like(w, dtype=torch.float32) for n, w in self.weights.items()}
        self.scan = _planned(sp.ScanPlan(self.tokens, channels, code))
        self.router = _planned(sp.RouterPlan(self.tokens, experts, k, code, renormalize=True))
        self.ortho = {n: _planned(sp.OrthoPlan(1, *w.shape, code)) for n, w in self.weights.items()}
        # what the ranks gather: summaries, counts, rows of a gradient
        self.gather_summary = sp.Plan(P, 2 * channels * 4)
        self.gather_counts = sp.Plan(P, (experts + 1) * 4)
        self.gather_rows = {n: sp.Plan(P, w.numel() // P * w.element_size()) for n, w in self.weights.items()}

        def new(*shape, dt=torch.float32):
            return torch.empty(*shape, dtype=dt, device="cuda")

        self.summary, self.summaries = new(P, 2, channels), new(P, P, 2, channels)
        self.first, self.last = new(P, channels), new(P, channels)
        self.carry = new(max(1, self.scan.carry_bytes), dt=torch.uint8)
        self.y, self.dgx = new(T, channels, dt=dtype), new(T, 2 * channels, dt=dtype)
        self.indices, self.chosen, self.lse = new(T, k, dt=torch.int32), new(T, k), new(T)
        self.counts, self.all_counts = new(P, experts + 1, dt=torch.int32), new(P, P, experts + 1, dt=torch.int32)
        self.sums, self.loss = new(P, experts + 1), new(P)
        self.dlogits = new(T, experts, dt=dtype)

    def run(self, h, dchosen, mask=None):
        """One step on h [T][width]; dchosen [T][k]: gradient that comes back from the chosen experts.
        Returns the balance loss of the whole batch and the gradients of the weights."""
        stream, c = torch.cuda.current_stream(), self.channels
        at = dict(gate_ld=2 * c, x_ld=2 * c, stream=stream)
        gx = h @ self.weights["in"]
        gate, x = gx[:, :c], gx[:, c:]
        # what each slice does to a state, everybody's, where each slice starts, the states
        self.scan.forward(gate, x, None, summary=self.summary, **at)
        self.gather_summary.allgather(self.summary, self.summaries, stream=stream)
        sp.scan_join(self.P, c, self.summaries, self.first, stream=stream)
        self.scan.forward(gate, x, self.y, h0=self.first, carry=self.carry, **at)
        # experts of every token, everybody's counts, the balance loss and its gradient
        logits = self.y @ self.weights["router"]
        self.router.forward(logits, self.indices, self.chosen, self.lse, self.counts, self.sums, mask=mask,
                            stream=stream)
        self.gather_counts.allgather(self.counts, self.all_counts, stream=stream)
        self.router.balance(self.all_counts, self.P, self.sums, self.loss, alpha=self.alpha, beta=self.beta,
                            stream=stream)
        self.router.backward(logits, self.indices, self.chosen, self.lse, self.all_counts, self.P, self.dlogits,
                             dweights=dchosen, alpha=self.alpha, beta=self.beta, mask=mask, stream=stream)
        # back through the recurrence, against time
        dy = self.dlogits @ self.weights["router"].T
        dgate, dx = self.dgx[:, :c], self.dgx[:, c:]
        self.scan.backward(gate, None, None, dy, None, None, dsummary=self.summary, gate_ld=2 * c, stream=stream)
        self.gather_summary.allgather(self.summary, self.summaries, stream=stream)
        sp.scan_join(self.P, c, self.summaries, self.last, reverse=True, stream=stream)
        self.scan.backward(gate, x, self.carry, dy, dgate, dx, dlast=self.last, dgate_ld=2 * c, dx_ld=2 * c, **at)
        # gradients: summed over the ranks, each of which owns a block of rows (one GPU: one product)
        grads = {"in": h.T @ self.dgx, "router": self.y.T @ self.dlogits}
        for name, w in self.weights.items():
            rows = grads[name].contiguous()
            full = torch.empty(self.P, *w.shape, dtype=self.dtype, device="cuda")
            self.gather_rows[name].allgather(rows, full, stream=stream)
            # every rank holds the whole gradient now; on one GPU the first one's copy stands for all
            self.ortho[name].muon_step(full[0], self.momentum[name], self.momentum[name], w, w, weight_dtype=self.code,
                                       lr=self.lr, weight_decay=0.01, scale=0.2 * math.sqrt(max(w.shape)), stream=stream)
        return self.loss.sum(), grads

    def status(self) -> None:
        """Waits, and raises where a wait inside a kernel gave up."""
        plans = [self.scan, *self.ortho.values(), self.gather_summary, self.gather_counts, *self.gather_rows.values()]
        if any(p.status() != sp.OK for p in plans):
            raise RuntimeError("a device-side wait timed out")


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--ranks", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=16384)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--channels", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--k", type=int, default=6)
    ap.add_argument("--steps", type=int, default=5)
    a = ap.parse_args()
    each = [a.tokens // a.ranks + (r < a.tokens % a.ranks) for r in range(a.ranks)]
    step = ShardedStep(each, a.width, a.channels, a.experts, a.k)
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(a.tokens, a.width, generator=g, device="cuda").bfloat16()
    dchosen = torch.randn(a.tokens, a.k, generator=g, device="cuda") * 1e-3
    for i in range(a.steps):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        loss, _ = step.run(h, dchosen)
        end.record()
        step.status()
        spread = step.counts[:, :-1].sum(0).float()
        print(f"step {i}: balance loss {loss.item():.6f}, busiest expert {spread.max().item() / spread.mean().item():.2f} "
              f"times the mean, {start.elapsed_time(end):.2f} ms")


if __name__ == "__main__":
    main()
