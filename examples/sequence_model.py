#!/usr/bin/env python3
"""A small sequence model trained by K workers through the coded exchange, with everything a worker does between its backward
pass and CODE o Q on the library's own kernels.

The task: position i of a random token sequence has to name the token `lag` places before it, which one attention layer
learns through its relative position bias.  The model's parameters are runs of the iterate X [d]; per half-step every worker
  - normalises its activations (layer norm) and biases its attention scores (causal buckets of the relative position),
  - writes the gradients of the norm's weight and bias and of the bias' table straight into its row of V [K][d],
  - clips all its gradients, the matrices' among them, to one global norm, gathered into V,
and the workers' rows are quantised, coded, decoded, averaged and stepped by the two extra-gradient half-steps.
The matrix products are torch's.

    python examples/sequence_model.py --steps 200
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2308_09187_amd import qgx, synth  # noqa: E402


class Model:
    """Runs of X, one after the other (multiples of 4 coordinates), and one step's forward and backward pass for K workers."""

    def __init__(self, vocabulary=16, width=32, heads=2, table=8, far=16, length=24):
        self.n, self.D, self.H, self.L, self.R = vocabulary, width, heads, length, table
        self.sizes = dict(norm_w=(width,), norm_b=(width,), table=(table, heads), wq=(width, width), wk=(width, width),
                          wv=(width, width), head=(width, vocabulary))
        self.at, self.d = {}, 0
        for name, shape in self.sizes.items():
            self.at[name] = self.d
            self.d += (math.prod(shape) + 3) // 4 * 4
        # causal: distances 0 .. 3 have a bucket each, further ones share four by their logarithm
        self.buckets = qgx.Buckets.logarithmic(table, far)

    def run_of(self, x, name):
        """A parameter in X [d], or every worker's gradient of it in V [K, d]."""
        shape = self.sizes[name]
        part = x[..., self.at[name]:self.at[name] + math.prod(shape)]
        return part.unflatten(-1, shape) if len(shape) > 1 else part

    def initial(self, generator):
        X = torch.zeros(self.d, device="cuda")
        self.run_of(X, "norm_w").fill_(1.0)
        for name in ("wq", "wk", "wv", "head"):
            w = self.run_of(X, name)
            w.copy_(torch.randn(w.shape, generator=generator, device="cuda") / math.sqrt(self.D))
        return X

    def gradients(self, ctx, X, V, embedding, tokens, targets):
        """tokens, targets [K, B, L].  Writes the runs of V that the library's kernels make; returns the mean loss and the
        matrices' gradients by name, [K, n] each."""
        K, B, L, D, H = *tokens.shape, self.D, self.H
        p = {name: self.run_of(X, name) for name in self.sizes}
        x0 = embedding[tokens].view(K, B * L, D)
        x, mean, rstd = ctx.layer_norm(x0, p["norm_w"], p["norm_b"])

        def heads(t):                                     # [K, B L, D] -> [K, B, H, L, D / H]
            return t.view(K, B, L, H, D // H).transpose(2, 3)

        def flat(t):
            return t.transpose(2, 3).reshape(K, B * L, D)

        q, k, v = heads(x @ p["wq"]), heads(x @ p["wk"]), heads(x @ p["wv"])
        scale = 1.0 / math.sqrt(D // H)
        scores = ctx.add_position_bias((q @ k.transpose(-1, -2)).mul_(scale), p["table"], self.buckets)
        attention = torch.softmax(scores, -1)
        mixed = flat(attention @ v)
        logits = mixed @ p["head"]
        logp = torch.log_softmax(logits, -1).view(K, B * L, self.n)
        seen = targets.view(K, B * L) >= 0
        t = targets.view(K, B * L).clamp_min(0)
        count = seen.sum(1).clamp_min(1).view(K, 1, 1)
        loss = -(logp.gather(2, t.unsqueeze(2)).squeeze(2) * seen).sum(1) / count.view(K)

        dlogits = (torch.exp(logp) - torch.nn.functional.one_hot(t, self.n)) * seen.unsqueeze(2) / count
        g = {"head": mixed.transpose(1, 2) @ dlogits}
        dmixed = heads(dlogits @ p["head"].t())
        dattention = dmixed @ v.transpose(-1, -2)
        dv = flat(attention.transpose(-1, -2) @ dmixed)
        dscores = attention * (dattention - (attention * dattention).sum(-1, keepdim=True))
        ctx.position_bias_backward(dscores, self.buckets, self.run_of(V, "table"))
        dq, dk = flat(dscores @ k).mul_(scale), flat(dscores.transpose(-1, -2) @ q).mul_(scale)
        xt = x.transpose(1, 2)
        g["wq"], g["wk"], g["wv"] = xt @ dq, xt @ dk, xt @ dv
        dx = dq @ p["wq"].t() + dk @ p["wk"].t() + dv @ p["wv"].t()
        ctx.layer_norm_backward(dx, x0, p["norm_w"], mean, rstd, dw=self.run_of(V, "norm_w"), db=self.run_of(V, "norm_b"),
                                need_dx=False)            # (the embedding is not learned)
        return loss.mean(), {name: t.reshape(K, -1) for name, t in g.items()}


class Trainer:
    def __init__(self, K=4, batch=8, lag=3, max_norm=0.25, seed=0, model=None):
        self.model, self.K, self.batch, self.lag, self.max_norm = model or Model(), K, batch, lag, max_norm
        m = self.model
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.embedding = torch.randn(m.n, m.D, generator=self.gen, device="cuda")
        self.X = m.initial(self.gen)
        self.half = torch.empty_like(self.X)
        self.V = torch.zeros(K, m.d, device="cuda")
        self.ctx = qgx.Context(m.d, K, 256, seed=seed)
        self.ctx.set_levels(synth.levels_exponential(16))
        self.ctx.state_init(self.X)
        self.streams = [self.ctx.new_stream(), self.ctx.new_stream()]
        # the matrices' gradients have buffers of their own; the others are runs of V as they stand
        self.matrices = {name: torch.empty(K, math.prod(m.sizes[name]), device="cuda") for name in ("wq", "wk", "wv", "head")}
        tensors = [self.matrices.get(name, self.V[:, m.at[name]:m.at[name] + math.prod(shape)]) for name, shape in m.sizes.items()]
        self.list = self.ctx.tensor_list(tensors, [m.at[name] for name in m.sizes])
        self.calls = 0

    def data(self):
        m = self.model
        tokens = torch.randint(0, m.n, (self.K, self.batch, m.L), generator=self.gen, device="cuda")
        targets = torch.full_like(tokens, -1)
        targets[..., self.lag:] = tokens[..., :-self.lag]
        return tokens, targets

    def dual_vectors(self, X):
        """The workers' clipped gradients at X in V, and their mean loss."""
        loss, g = self.model.gradients(self.ctx, X, self.V, self.embedding, *self.data())
        for name, buffer in self.matrices.items():
            buffer.copy_(g[name])
        self.ctx.clip_gradients(self.list, self.max_norm, out=self.V)
        return loss

    def step(self):
        """One iteration: two rounds of gradients, coded exchange and half-step.  Returns the loss at its first point."""
        first, second = self.streams
        loss = self.dual_vectors(self.X)
        self.ctx.quantize_encode(self.V, self.calls, first)
        self.ctx.eg_step(0, first, None, self.half)
        self.dual_vectors(self.half)
        self.ctx.quantize_encode(self.V, self.calls + 1, second)
        self.ctx.eg_step(1, second, first, self.X)
        self.calls += 2
        return loss


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--K", type=int, default=4)
    a = ap.parse_args()
    trainer = Trainer(K=a.K)
    for i in range(a.steps):
        loss = trainer.step()
        if i % 25 == 0 or i + 1 == a.steps:
            print("step %4d  loss %.4f  (chance %.4f)  gamma %.4f" % (i, loss.item(), math.log(trainer.model.n), trainer.ctx.scalars()["gamma"]), flush=True)
    assert trainer.ctx.poll_error() == 0


if __name__ == "__main__":
    main()
