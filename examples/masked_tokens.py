"""Masked token prediction on program-shaped graphs: the token operators around a GGNN.

Every node carries a token of a vocabulary of V; 15% of them are hidden behind a mask token and are
to be predicted from the graph around them.  One [V + 1, H] table serves both ends:

    ids -> embed_fwd (scaled, dropout) -> ggnn_step (T steps) -> dropout_fwd -> xent_fwd: loss
    xent_bwd -> dropout_bwd -> ggnn_step_bwd -> embed_bwd (added to the table's gradient) -> adam_step

The masks of the two dropouts are never stored: the backward calls pass their forward calls' (seed,
call).  Tokens run along each graph's chain edges (the next node's token is the last one's plus one), so
a hidden token follows from a neighbour and the loss falls from log V.

    python examples/masked_tokens.py [--steps 120]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1906_11786_gb300 import lib as L  # noqa: E402
from paper_1906_11786_gb300 import synth  # noqa: E402

WEIGHTS = ("W", "W_ih", "W_hh")  # bf16 working copies; the biases stay fp32


def chain_tokens(graph, vocab, rng):
    """Token of every node: one more (mod vocab) than that of the node before it on the chain."""
    nxt = np.full(graph.n_nodes, -1)
    chain = graph.etype == 0
    nxt[graph.src[chain]] = graph.dst[chain]
    first = np.setdiff1d(np.arange(graph.n_nodes), graph.dst[chain])[0]
    tokens, at, t = np.zeros(graph.n_nodes, np.int64), first, int(rng.integers(vocab))
    while at >= 0:
        tokens[at] = t % vocab
        at, t = nxt[at], t + 1
    return tokens


class MaskedTokenModel:
    """One packed batch, its GGNN and tied table, with every buffer allocated once."""

    def __init__(self, vocab=60, H=64, T=2, p=0.1, seed=1906):
        self.V, self.H, self.T, self.p, self.seed = vocab, H, T, p, seed
        P, S = 6, 64
        graphs = synth.gen_batch(16, 100, 300, 3, True, 16, 16, 1.0, seed)
        self.plan = L.band_plan(graphs, P, S)
        self.plan.upload()
        info = self.plan.info()
        self.N, self.n_real = info["n_pad"], info["n_real"]
        rng = np.random.default_rng(seed)
        # tokens in band order; padding rows carry none
        tokens = np.concatenate([chain_tokens(g, vocab, rng) for g in graphs])
        self.tokens = np.full(self.N, -1, np.int32)
        self.tokens[:self.n_real] = tokens[self.plan.export(L.BG_EXPORT_GATHER)]
        prm = synth.gen_params(P, H, seed + 1, mean_in_degree=info["n_kept"] / info["n_real"])
        prm.pop("w_out")
        prm["table"] = rng.standard_normal((vocab + 1, H)) / np.sqrt(H)  # the last row is the mask token
        f32 = {k: torch.from_numpy(np.asarray(v, np.float32)).cuda() for k, v in prm.items()}
        self.master = f32
        self.work = {k: v.to(torch.bfloat16) if k in WEIGHTS + ("table",) else v
                     for k, v in f32.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in f32.items()}
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in f32.items()}

        def bf16():
            return torch.empty(self.N, H, device="cuda", dtype=torch.bfloat16)

        def scratch(n):
            return torch.empty(max(n, 256), device="cuda", dtype=torch.uint8)

        self.E0, self.ET, self.X = bf16(), bf16(), bf16()
        self.dX, self.dE0 = (torch.empty(self.N, H, device="cuda") for _ in range(2))
        self.loss, self.lse = (torch.empty(self.N, device="cuda") for _ in range(2))
        self.saved = scratch(L.ggnn_saved_bytes(self.plan, "bf16", H, T))
        self.ws = scratch(max(
            [L.ggnn_workspace_bytes(self.plan, "bf16", H, T, op)
             for op in (L.BG_OP_GGNN_FWD, L.BG_OP_GGNN_BWD)] +
            [L.xent_workspace_bytes("bf16", self.N, H, vocab + 1, op)
             for op in (L.BG_OP_XENT_FWD, L.BG_OP_XENT_BWD)] +
            [L.embed_workspace_bytes(self.N, H, vocab + 1)]))
        self.call = 0

    def hide(self, rng):
        """(ids, targets, gradient of the mean loss) of a step that hides 15% of the tokens."""
        hidden = (rng.random(self.N) < 0.15) & (self.tokens >= 0)
        ids = np.where(hidden, self.V, self.tokens).astype(np.int32)
        target = np.where(hidden, self.tokens, -1).astype(np.int32)
        dloss = np.full(self.N, 1.0 / max(int(hidden.sum()), 1), np.float32)
        return (torch.from_numpy(x).cuda() for x in (ids, target, dloss))

    def loss_and_gradients(self, ids, target, dloss):
        """Fills self.grad; the loss of each hidden node is in self.loss, 0 elsewhere."""
        w, scale = self.work, float(np.sqrt(self.H))
        enter, leave = 2 * self.call, 2 * self.call + 1  # a `call` of its own for each dropout
        self.call += 1
        drop = dict(p=self.p, seed=self.seed)
        L.embed_fwd("bf16", ids, w["table"], self.E0, scale=scale, call=enter, **drop)
        L.ggnn_step(self.plan, "bf16", self.H, self.T, w, self.E0, self.ET, self.saved, self.ws)
        L.dropout_fwd("bf16", self.ET, self.X, call=leave, **drop)
        L.xent_fwd("bf16", self.X, w["table"], target, self.loss, self.lse, self.ws)
        L.xent_bwd("bf16", self.X, w["table"], target, self.lse, dloss, "f32", self.dX,
                   self.grad["table"], self.ws)
        L.dropout_bwd(self.dX, self.dX, call=leave, **drop)
        g = {"d" + k: v for k, v in self.grad.items()}
        L.ggnn_step_bwd(self.plan, "bf16", self.H, self.T, w, self.saved, self.dX, self.dE0, g,
                        self.ws)
        L.embed_bwd(ids, self.dE0, self.grad["table"], self.ws, scale=scale, call=enter,
                    flags=L.BG_ACCUM, **drop)

    def update(self, step, lr):
        for k, master in self.master.items():
            m, v = self.moments[k]
            work = self.work[k] if self.work[k] is not master else None
            L.adam_step(master, work, m, v, self.grad[k], lr, 0.9, 0.999, 1e-8, step)


def train(steps=120, lr=3e-3, report=None, **model):
    """Mean loss of the hidden nodes at each step."""
    net = MaskedTokenModel(**model)
    rng = np.random.default_rng(7)
    losses = []
    for step in range(1, steps + 1):
        ids, target, dloss = net.hide(rng)
        net.loss_and_gradients(ids, target, dloss)
        net.update(step, lr)
        losses.append(float(net.loss.sum()) / max(int((target >= 0).sum()), 1))
        if report and (step == 1 or step % report == 0):
            print(f"step {step:4d}  loss {losses[-1]:.3f}", flush=True)
    L.check_device()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=120)
    train(ap.parse_args().steps, report=10)
