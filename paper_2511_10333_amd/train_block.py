"""A data-parallel training step around the compressor, on one GPU: a stack of residual gated feed-forward blocks.

    python -m paper_2511_10333_amd.train_block --layers 4 --hidden 512 --ff 2048 --tokens 1024 --steps 40

Per step: the norm before the first block; per block the gated feed-forward block and the norms after it and before the next,
with gate and residual scale; the backward passes, which leave the weight gradients in the compressor's tensors; the entropy of
those gradients and, per window, the rank; compress and decompress with error feedback (a job of several ranks all-reduces P and
Q between the two phases of the compress); the global norm and clipping; a momentum update.  The model learns the outputs of
another one of the same shape.  Prints one JSON line per window.  Needs a GPU and the built library.
"""
from __future__ import annotations

import argparse
import json
import math

import torch

from . import Context, FeedForward, PreparedBatch, RankParams, RankState, Tensor, select_rank, tensor_bypassed

RANKS = [4, 8, 16, 32, 64]
CHUNK, STRIDE, BINS = 64, 100, 1024


def reference_shape(shapes):
    """The shape that the rank rule's error function is evaluated at: the smallest matrix that is compressed at every rank.  (Where a
    model has none, a square of twice the largest rank, so that the rule still answers.)"""
    r = max(RANKS)
    matrices = [tuple(s) for s in shapes if len(s) == 2 and min(s) >= r and not tensor_bypassed(*s, r)]
    return min(matrices, key=lambda s: s[0] * s[1], default=(2 * r, 2 * r))


class Model:
    """Weights of ``layers`` blocks, their gradients, and the two passes through them."""

    def __init__(self, ctx: Context, layers: int, hidden: int, ff: int, tokens: int, sequence: int, dtype=torch.float32,
                 act: str = "silu", seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s, std=1.0, mean=0.0: (mean + std * torch.randn(*s, generator=g, device="cuda")).to(dtype)
        self.ctx, self.hidden, self.ff, self.tokens, self.sequence = ctx, hidden, ff, tokens, sequence
        self.scale = 1.0 / math.sqrt(layers)
        gates = -(-tokens // sequence)
        self.blocks = [{"w_gate": randn(ff, hidden, std=hidden ** -0.5), "w_up": randn(ff, hidden, std=hidden ** -0.5),
                        "w_down": randn(hidden, ff, std=ff ** -0.5), "w_pre": randn(hidden, std=0.02, mean=1.0),
                        "w_post": randn(hidden, std=0.02, mean=1.0), "gate": randn(gates, hidden, std=0.1, mean=1.0)}
                       for _ in range(layers)]
        self.w_last = randn(hidden, std=0.02, mean=1.0)         # of the norm after the last block
        self.grads = [{k: torch.zeros_like(w) for k, w in b.items()} for b in self.blocks]
        self.g_last = torch.zeros_like(self.w_last)
        self.weights = [FeedForward(b["w_gate"], b["w_up"], b["w_down"], act) for b in self.blocks]
        act_of = lambda *s: torch.empty(s, device="cuda", dtype=dtype)
        stat = lambda: torch.empty(tokens, device="cuda")
        # what the forward pass keeps: per block its input's sum and norm, the projections, its output and two row statistics
        self.kept = [{"n": act_of(tokens, hidden), "g": act_of(tokens, ff), "u": act_of(tokens, ff), "y": act_of(tokens, hidden),
                      "x": act_of(tokens, hidden), "r_pre": stat(), "r_post": stat()} for _ in range(layers)]
        self.n_last, self.x_last, self.r_last = act_of(tokens, hidden), act_of(tokens, hidden), stat()
        self.d = {k: act_of(tokens, hidden) for k in ("x", "n", "y")}
        ctx.reserve_ff(dtype, tokens, hidden, ff, backward=True)
        ctx.reserve_block_norm(tokens, hidden)

    def parameters(self):
        """Pairs of weight and gradient."""
        return [(b[k], g[k]) for b, g in zip(self.blocks, self.grads) for k in b] + [(self.w_last, self.g_last)]

    def _after(self, i):
        """The norm that follows block i: its weight, its output, the sum and the statistic."""
        if i + 1 < len(self.blocks):
            k = self.kept[i + 1]
            return self.blocks[i + 1]["w_pre"], k["n"], k["x"], k["r_pre"]
        return self.w_last, self.n_last, self.x_last, self.r_last

    def forward(self, x):
        c, k = self.ctx, self.kept[0]
        c.block_norm_forward(x, None, None, None, self.blocks[0]["w_pre"], k["x"], k["n"], None, k["r_pre"])
        for i, (b, k) in enumerate(zip(self.blocks, self.kept)):
            c.ff_forward(self.weights[i], k["n"], k["y"], k["g"], k["u"])
            w, n, x_next, r = self._after(i)
            c.block_norm_forward(k["x"], k["y"], b["w_post"], b["gate"], w, x_next, n, k["r_post"], r, scale=self.scale,
                                 rows_per_gate=self.sequence)
        return self.n_last

    def backward(self, dn):
        """From the gradient of what forward() returned; leaves the weights' gradients in ``grads``.  Returns that of x."""
        c, d = self.ctx, self.d
        d["n"].copy_(dn)
        d["x"].zero_()
        for i in reversed(range(len(self.blocks))):
            b, g, k = self.blocks[i], self.grads[i], self.kept[i]
            w, _, x_next, r = self._after(i)
            dw = self.grads[i + 1]["w_pre"] if i + 1 < len(self.blocks) else self.g_last
            c.block_norm_backward(d["x"], d["n"], x_next, k["y"], b["w_post"], b["gate"], w, k["r_post"], r, d["x"], d["y"],
                                  g["w_post"], g["gate"], dw, scale=self.scale, rows_per_gate=self.sequence)
            c.ff_backward(self.weights[i], k["n"], k["g"], k["u"], d["y"], d["n"], g["w_gate"], g["w_up"], g["w_down"])
        k = self.kept[0]
        c.block_norm_backward(d["x"], d["n"], k["x"], None, None, None, self.blocks[0]["w_pre"], None, k["r_pre"], d["x"], None,
                              None, None, self.grads[0]["w_pre"])
        return d["x"]


class Step:
    """What follows the backward pass: entropy, rank, compress and decompress with error feedback, clipping, update."""

    def __init__(self, model: Model, max_norm: float, lr: float, momentum: float, seed: int = 0):
        self.m, self.ctx, self.max_norm, self.lr, self.momentum = model, model.ctx, max_norm, lr, momentum
        self.pairs = model.parameters()
        self.velocity = [torch.zeros_like(w) for w, _ in self.pairs]
        self.sent = [torch.empty_like(g) for _, g in self.pairs]
        r = max(RANKS)
        self.tensors = []
        for i, ((_, g), out) in enumerate(zip(self.pairs, self.sent)):
            if g.dim() == 1 or min(g.shape) == 1 or tensor_bypassed(*g.shape, min(RANKS)):
                self.tensors.append(Tensor(g, out))
                continue
            m, n = g.shape
            Q = torch.empty((n, r), device="cuda")
            self.ctx.init_q(Q, 0, r, seed + i)
            self.tensors.append(Tensor(g, out, torch.zeros((m, n), device="cuda"), Q, torch.empty((m, r), device="cuda"), True))
        self.ctx.reserve_batch([tuple(t.grad.shape) if t.grad.dim() == 2 else (1, t.grad.numel()) for t in self.tensors])
        self.batch = PreparedBatch(self.tensors)
        self.clip = PreparedBatch([Tensor(o, o) for o in self.sent])
        self.norm_coef = torch.zeros(2, device="cuda")
        flats = [g.view(-1) for _, g in self.pairs if g.dim() == 2]
        self.flats = flats[:32]                                # one estimate takes up to 32 buffers

    def entropy(self, step: int) -> float:
        return self.ctx.entropy_estimate(self.flats, STRIDE, CHUNK, 7, step, BINS).h_diff_nats

    def update(self, rank: int) -> None:
        """rank 0: the gradients as they are (the warm-up)."""
        c = self.ctx
        if rank:
            c.compress_batch(self.batch, rank)
            c.decompress_batch(self.batch, rank)
            for t in self.tensors:
                t.residual_is_zero = False
        else:
            torch._foreach_copy_(self.sent, [g for _, g in self.pairs])
        c.grad_sumsq_batch(self.clip)
        c.clip_batch(self.clip, self.max_norm, self.norm_coef)
        torch._foreach_mul_(self.velocity, self.momentum)
        torch._foreach_add_(self.velocity, self.sent)
        torch._foreach_add_([w for w, _ in self.pairs], self.velocity, alpha=-self.lr)


def train(layers=4, hidden=512, ff=2048, tokens=1024, sequence=256, steps=40, window=5, dtype=torch.float32, lr=0.5, momentum=0.9,
          max_norm=1.0, seed=0, report=None):
    """Trains and returns the losses; ``report``: called with a dict per window."""
    ctx = Context(0, max_bins=BINS, max_rank=max(RANKS), max_rows=64, max_cols=64)
    teacher = Model(ctx, layers, hidden, ff, tokens, sequence, dtype, seed=seed + 1)
    model = Model(ctx, layers, hidden, ff, tokens, sequence, dtype, seed=seed + 2)
    step = Step(model, max_norm, lr, momentum)
    state = RankState()
    prm = RankParams(*reference_shape([w.shape for w, _ in step.pairs]), min(RANKS), max(RANKS), allowed=RANKS, total_iters=steps)
    g = torch.Generator(device="cuda").manual_seed(seed)
    losses, entropies, rank = [], [], 0
    for i in range(steps):
        x = torch.randn(tokens, hidden, generator=g, device="cuda").to(dtype)
        target = teacher.forward(x).clone()
        diff = (model.forward(x).float() - target.float())
        losses.append(float(0.5 * diff.square().sum(1).mean()))
        model.backward((diff / tokens).to(dtype))
        entropies.append(step.entropy(i))
        step.update(rank)
        if len(entropies) == window:
            rank = select_rank(state, entropies, window, prm).rank
            if report:
                norm, coef = step.norm_coef.tolist()
                report({"step": i + 1, "loss": losses[-1], "entropy": sum(entropies) / window, "rank": rank, "grad_norm": norm,
                        "clip": coef})
            entropies = []
    torch.cuda.synchronize()
    ctx.close()
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 4), ("hidden", 512), ("ff", 2048), ("tokens", 1024), ("sequence", 256), ("steps", 40), ("window", 5)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    losses = train(a.layers, a.hidden, a.ff, a.tokens, a.sequence, a.steps, a.window, torch.float32 if a.dtype == "f32" else torch.bfloat16,
                   lr=a.lr, report=lambda d: print(json.dumps(d), flush=True))
    print(json.dumps({"first_loss": losses[0], "last_loss": losses[-1]}))


if __name__ == "__main__":
    main()
