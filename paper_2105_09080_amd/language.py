"""A small language model trained by Gossip-PGA on n nodes: the operators of language models run together.

Every node predicts the next token of its own text from the last two, with its own parameters x_i, a row of X:

    a = sqrt(D) E_i[token[t]],  b = sqrt(D) F_i[token[t-1]]           two embedding tables of V rows (padding before the first)
    y = layer norm of (b + dropout(a)), with gamma_i and beta_i
    v = y + Wd_i (act(Wg_i y) * Wu_i y)                               with ff > 0 hidden units; v = y without
    z = v E_i^T                                                       the output layer is the first table again
    f_i = mean cross-entropy of softmax(z) against token[t+1]

The backward pass writes G column block by column block: the output layer's gradient of E_i first, the embedding's is added
to it.  With ``orthogonal`` the feed-forward block's three gradients become orthogonalised updates in their place.  Then gpga_step
(or gpga_aga_step, which takes the nodes' losses as they are) updates and mixes.  Everything but the two products with E is the
library's; the products are the caller's own, in torch.

    python -m paper_2105_09080_amd.language --n 16 --iters 300
    python -m paper_2105_09080_amd.language --n 16 --iters 300 --ff 384 --orthogonal
"""
from __future__ import annotations

import argparse
import json
import math
import time

import numpy as np
import torch

from . import binding as B
from . import inputs
from .harness import Simulation


class NextTokenModel:
    """The model above on a simulation's rows.  ``dtype``: type of the activations between the operators."""

    def __init__(self, n: int, V: int, D: int, *, topology: str = "ring", H: int = 8, lr: float = 0.5, momentum: float = 0.9,
                 p: float = 0.1, seed: int = 0, dtype: torch.dtype = torch.float32, stream=None, ff: int = 0,
                 act: str = "silu", orthogonal: bool = False):
        self.n, self.V, self.D, self.p, self.seed, self.dtype = n, V, D, p, seed, dtype
        self.ff, self.act, self.orthogonal = ff, act, orthogonal and ff > 0
        self.E, self.F = 0, V * D                                   # column offsets
        self.gamma, self.beta = 2 * V * D, 2 * V * D + D
        self.scale = math.sqrt(D)
        after = 2 * V * D + 2 * D
        self.gate, self.up, self.down = after, after + ff * D, after + 2 * ff * D
        x0 = inputs.initial_point(after + 3 * ff * D, seed) / self.scale
        x0[self.gamma:self.beta], x0[self.beta:after] = 1.0, 0.0
        self.sim = Simulation(n, x0.size, topology=topology, H=H, lr=lr, momentum=momentum, x0=x0, stream=stream)

    def table(self, rows: torch.Tensor) -> torch.Tensor:
        """(n, V, D) view of the first table's columns of X or G."""
        return rows[:, self.E:self.E + self.V * self.D].unflatten(1, (self.V, self.D))

    def forward(self, tokens, previous, labels, p: float, grad: bool):
        s = self.sim
        a = s.embed(tokens, self.E, self.V, self.D, scale=self.scale, dtype=self.dtype)
        b = s.embed(previous, self.F, self.V, self.D, scale=self.scale, dtype=self.dtype)
        y, u, stats = s.layer_norm(a, self.gamma, self.beta, residual=b, p=p, seed=self.seed)
        v, hidden = y, None
        if self.ff:
            h, hidden = s.gated_ff(y, self.gate, self.up, self.down, self.ff, act=self.act, keep=grad)
            v = y + h
        table = self.table(s.X)
        z = torch.bmm(v.float(), table.transpose(1, 2).contiguous()).to(self.dtype)
        loss, dz = s.token_loss(z, labels, grad=z if grad else False)   # the gradient takes the logits' place
        return loss, dz, v, y, hidden, u, stats, table

    def gradients(self, tokens, previous, labels) -> torch.Tensor:
        """Losses of the nodes; their gradients in G."""
        s = self.sim
        with torch.cuda.stream(s.stream):
            loss, dz, v, y, hidden, u, stats, table = self.forward(tokens, previous, labels, self.p, True)
            dz = dz.float()
            self.table(s.G).copy_(torch.bmm(dz.transpose(1, 2).contiguous(), v.float()))
            dy = torch.bmm(dz, table.contiguous()).to(self.dtype)
            if self.ff:
                dy = dy + s.gated_ff_grad(dy, y, hidden, self.gate, self.up, self.down, act=self.act)
                if self.orthogonal:
                    s.orthogonalize(self.gate, self.ff, self.D, count=2, scale=self.update_scale(self.ff, self.D))
                    s.orthogonalize(self.down, self.D, self.ff, scale=self.update_scale(self.D, self.ff))
            du, dx = s.layer_norm_grad(dy, u, stats, self.gamma, self.beta, p=self.p, seed=self.seed)
            s.embed_grad(tokens, dx, self.E, self.V, scale=self.scale, accumulate=True)
            s.embed_grad(previous, du, self.F, self.V, scale=self.scale)
        return loss

    @staticmethod
    def update_scale(rows: int, cols: int) -> float:
        """An orthogonalised rows x cols update has about min(rows, cols) singular values of 1: elements of root mean square 0.02."""
        return 0.02 * math.sqrt(max(rows, cols))

    def losses(self, tokens, previous, labels) -> torch.Tensor:
        """Losses without dropout and without gradients."""
        with torch.cuda.stream(self.sim.stream):
            return self.forward(tokens, previous, labels, 0.0, False)[0]

    def batches(self, text: np.ndarray):
        """(iters, n, T) int32 tables on the device from (iters, n, sequences, length + 1) text: tokens, the tokens before
        them (-1 before the first of a sequence), the tokens after them."""
        iters, n, _, _ = text.shape
        previous = np.concatenate([np.full_like(text[..., :1], -1), text[..., :-2]], axis=3)
        return [self.sim.upload_batches(t.reshape(iters, n, -1)) for t in (text[..., :-1], previous, text[..., 1:])]


def train(model: NextTokenModel, text: np.ndarray, *, every: int = 50, adaptive: bool = False):
    """One pass over ``text``; yields a record every ``every`` iterations."""
    sim, iters = model.sim, text.shape[0]
    tables = model.batches(text)
    means = torch.empty(iters, dtype=torch.float64, device=sim.device)
    if adaptive:
        sim.aga_enable(4, iters // 10, 64)
    sim.stream.synchronize()
    began = time.perf_counter()
    for k in range(iters):
        loss = model.gradients(*(t[k] for t in tables))
        B.gpga_node_mean(sim.ctx, loss, means[k:])
        if adaptive:
            sim.aga_step(loss)
        else:
            sim.step()
        if (k + 1) % every == 0 or k + 1 == iters:
            sim.stream.synchronize()
            yield {"iteration": k + 1, "loss": float(means[k]), "consensus": sim.consensus_error(), "period": sim.period,
                   "iterations_per_s": (k + 1) / (time.perf_counter() - began)}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--n", type=int, default=16)
    ap.add_argument("--vocabulary", type=int, default=500)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--length", type=int, default=64)
    ap.add_argument("--iters", type=int, default=300)
    ap.add_argument("--topology", default="ring", choices=["ring", "grid", "expo", "expo1", "none", "full"])
    ap.add_argument("--H", type=int, default=8)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--dtype", default="bf16", choices=["f32", "bf16"])
    ap.add_argument("--ff", type=int, default=0, help="hidden units of a gated feed-forward block (0: none)")
    ap.add_argument("--activation", default="silu", choices=sorted(B.ACTIVATION))
    ap.add_argument("--orthogonal", action="store_true", help="orthogonalised updates of the feed-forward matrices")
    ap.add_argument("--adaptive", action="store_true", help="adaptive averaging period (Gossip-AGA)")
    args = ap.parse_args()
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[args.dtype]
    model = NextTokenModel(args.n, args.vocabulary, args.width, topology=args.topology, H=args.H, lr=args.lr, p=args.dropout,
                           dtype=dtype, ff=args.ff, act=args.activation, orthogonal=args.orthogonal)
    text = inputs.markov_text(args.iters, args.n, args.sequences, args.length, args.vocabulary)
    for record in train(model, text, adaptive=args.adaptive):
        print(json.dumps(record), flush=True)


if __name__ == "__main__":
    main()
