"""A transformer's training step out of ``ops``, as a program for the simulator.

    python -m paper_2006_09616_amd.step [--layers 4 --batch 8 --seq 512 --hidden 768 --heads 12 --vocab 32000]

runs the step, measures what each of its operators takes (microseconds,
forward and backward) and stores (bytes), simulates the resulting trace at
memory budgets down to where it no longer fits, and runs the step once more
with the layers' activations dropped and recomputed.

The step: embedding, layers of (norm, projection, attention, projection,
dropout with the residual sum, norm, two projections, dropout with the residual
sum), norm, logits, log probabilities of the next tokens.  Attention is causal
and within documents.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch
import torch.nn.functional as F

from . import dtr, ops
from . import workloads as W


class Step:
    """Parameters, one batch of tokens, and the step's operators in order."""

    def __init__(self, layers=4, batch=8, seq=512, hidden=768, heads=12, vocab=32000, p=0.1, cap=30.0, documents=2,
                 dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.layers, self.batch, self.seq, self.hidden, self.heads = layers, batch, seq, hidden, heads
        self.p, self.cap, self.seed = p, cap, seed

        def weight(*shape):
            return (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(device=device, dtype=dtype).requires_grad_()

        H = hidden
        self.weights = {"embedding": weight(vocab, H), "head": weight(vocab, H)}
        for i in range(layers):
            for name, shape in (("qkv", (3 * H, H)), ("proj", (H, H)), ("up", (4 * H, H)), ("down", (H, 4 * H))):
                self.weights[f"{name}{i}"] = weight(*shape)
        tokens = torch.randint(0, vocab, (batch, seq + 1), generator=g)
        cuts = torch.randint(1, seq, (batch, documents - 1), generator=g)
        self.docs = (torch.arange(seq)[None, :, None] >= cuts[:, None]).sum(2).to(torch.int32).to(device)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, heads + 1) / heads).to(device)
        self.tokens, self.targets = tokens[:, :-1].reshape(-1).to(device), tokens[:, 1:].reshape(-1).to(device)

    # the operators; each a function of its input tensors

    def norm(self, x):
        return F.layer_norm(x, (self.hidden,))

    def attend(self, qkv):
        q, k, v = qkv.view(self.batch, self.seq, 3, self.heads, -1).unbind(2)
        out = ops.attention(q, k, v, cap=self.cap, slopes=self.slopes, causal=True, docs=self.docs)
        return out.reshape(-1, self.hidden)

    def drop(self, x, residual, number):
        # every call has draws of its own; recomputed, it makes the same mask again
        return ops.dropout_add(x, residual, p=self.p, seed=self.seed, offset=number * (x.numel() // 2 + 1))

    def loss(self, logits):
        return -ops.token_logprobs(logits, self.targets).logp.mean()

    def program(self):
        """(name, function, inputs) of every operator; an input is the name of
        an operator before it."""
        w, prog = self.weights, [("x", lambda: F.embedding(self.tokens, w["embedding"]), [])]
        x = "x"
        for i in range(self.layers):
            def op(name, f, *ins, i=i):
                prog.append((f"{name}{i}", f, list(ins)))
                return f"{name}{i}"
            n = op("norm", self.norm, x)
            qkv = op("qkv", lambda t, i=i: t @ w[f"qkv{i}"].t(), n)
            att = op("attention", self.attend, qkv)
            pr = op("proj", lambda t, i=i: t @ w[f"proj{i}"].t(), att)
            mid = op("sum", lambda t, r, i=i: self.drop(t, r, 2 * i), pr, x)
            n = op("norm_b", self.norm, mid)
            up = op("up", lambda t, i=i: F.gelu(t @ w[f"up{i}"].t()), n)
            down = op("down", lambda t, i=i: t @ w[f"down{i}"].t(), up)
            x = op("sum_b", lambda t, r, i=i: self.drop(t, r, 2 * i + 1), down, mid)
        prog.append(("norm_end", self.norm, [x]))
        prog.append(("logits", lambda t: t @ w["head"].t(), ["norm_end"]))
        prog.append(("loss", self.loss, ["logits"]))
        return prog

    def run(self):
        """The step with every activation stored: the loss and the gradients of the weights."""
        made = {}
        for name, f, ins in self.program():
            made[name] = f(*(made[i] for i in ins))
        grads = torch.autograd.grad(made["loss"], list(self.weights.values()))
        return made["loss"].detach(), dict(zip(self.weights, grads))

    def run_rematerialized(self):
        """The same with only the layers' inputs stored: the operators of a
        layer run again before its backward pass.  The operators of ``ops``
        give the same bits again, so the gradients are those of ``run``."""
        prog = self.program()
        per = 9                                           # operators of a layer
        parts = [prog[:1]] + [prog[1 + per * i:1 + per * (i + 1)] for i in range(self.layers)] + [prog[1 + per * self.layers:]]
        weights = list(self.weights.values())

        def run_part(part, name, x):
            made = {name: x} if name else {}
            for n, f, ins in part:
                made[n] = f(*(made[i] for i in ins))
            return made[part[-1][0]]

        stored, x, name = [], None, None
        with torch.no_grad():
            for part in parts:
                stored.append((name, x))
                x, name = run_part(part, name, x), part[-1][0]
        loss, grad = x, None
        total = {k: None for k in self.weights}
        for part, (name, x) in reversed(list(zip(parts, stored))):
            x = x.detach().requires_grad_() if x is not None else None
            out = run_part(part, name, x)
            wanted = ([x] if x is not None else []) + weights
            got = torch.autograd.grad(out, wanted, grad, allow_unused=True)
            if x is not None:
                grad, got = got[0], got[1:]
            for k, g in zip(total, got):
                if g is not None:
                    total[k] = g if total[k] is None else total[k] + g
        return loss, total

    def measure(self, repeats=5):
        """(inputs, bytes, microseconds forward, microseconds backward) of every operator."""
        made, rows, index = {}, [], {}

        def timed(f):
            f()
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            for _ in range(repeats):
                f()
            end.record()
            end.synchronize()
            return max(1, round(start.elapsed_time(end) * 1000 / repeats))

        for n, (name, f, ins) in enumerate(self.program()):
            xs = [made[i].detach().requires_grad_() for i in ins]
            forward = timed(lambda: f(*xs))
            out = f(*xs)
            made[name], index[name] = out.detach(), n
            ones = torch.ones_like(out)
            leaves = xs or [self.weights["embedding"]]
            backward = timed(lambda: torch.autograd.grad(out, leaves, ones, retain_graph=True))
            rows.append(([index[i] for i in ins], out.numel() * out.element_size(), forward, backward))
        return rows

    def trace(self, repeats=5) -> W.Trace:
        """The step as an operator trace with measured costs (microseconds)."""
        rows = self.measure(repeats)
        off, flat = W._csr([r[0] for r in rows])
        return W.with_backward(off, flat, np.array([r[1] for r in rows], np.int64), np.array([r[2] for r in rows], np.int64),
                               np.array([r[3] for r in rows], np.int64)[::-1].copy(), name=f"step{self.layers}",
                               meta=dict(layers=self.layers, hidden=self.hidden, seq=self.seq, batch=self.batch))


def simulate(trace: W.Trace, percents=(100, 80, 60, 50, 40, 30, 25, 20), heuristics=(W.H_DTR, W.H_EQ, W.H_LRU)):
    """[(heuristic, percent, result record)] of the trace at shares of its peak."""
    peak = W.natural_peak(trace)
    rows = [(0, h, max(1, peak * p // 100), 1) for h in heuristics for p in percents]
    return list(zip([W.HEURISTIC_NAMES[r[1]] for r in rows], [p for _ in heuristics for p in percents],
                    dtr.run([trace], W.make_specs(rows))))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("layers", 4), ("batch", 8), ("seq", 512), ("hidden", 768), ("heads", 12), ("vocab", 32000)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args(argv)
    step = Step(**vars(a))
    loss, grads = step.run()
    print(f"loss {float(loss):.4f}")
    trace = step.trace()
    peak = W.natural_peak(trace)
    fwd = trace.n_ops // 2
    print(f"{trace.n_ops} operators, {int(trace.op_cost.sum())} us, peak {peak / 2**20:.0f} MiB; "
          f"scores, probabilities and masks that are not stored: "
          f"{a.layers * (2 * a.batch * a.heads * a.seq * a.seq * 2 + 2 * a.batch * a.seq * a.hidden) / 2**20:.0f} MiB")
    for h, pct, r in simulate(trace):
        what = f"{r['total_cost'] / r['base_cost']:.3f}x, {r['n_remats']} rematerializations" if r["status"] == 0 else "does not fit"
        print(f"  {h:4s} {pct:3d}% of the peak: {what}")
    again, regrads = step.run_rematerialized()
    same = torch.equal(again, loss) and all(torch.equal(grads[k], regrads[k]) for k in grads)
    print(f"layers dropped and recomputed: loss {float(again):.4f}, {'the same bits' if same else 'other bits'}; "
          f"{fwd} forward operators")


if __name__ == "__main__":
    main()
