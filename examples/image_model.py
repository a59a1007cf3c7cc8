#!/usr/bin/env python3
"""A small image model trained by K workers through the coded exchange, its backward pass working from activations kept in 8 bits.

The task: every place of an image of random tokens has to name the token that lies `shift` rows and columns further on, which one attention layer
learns through rotary positions with two axes.  The model's parameters are runs of the iterate X [d]; per half-step every worker
  - normalises its images by groups of channels with an activation, keeping the input in 8 bits in the same pass,
  - keeps what the linear layers take in 8 bits as well, rounded without bias, each tensor by draws of its own (so that their weight gradients, which are
    linear in it, have the expectation of the exact ones, as the method asks of its oracle; the norm's, of its own kept input, are not linear in that
    and are off the exact ones by the order of a step squared in expectation),
  - turns queries and keys by their places' rows and columns,
  - writes all gradients, the matrices' from the matrix cores, straight into its row of V [K][d], where they are clipped to one global norm,
and the workers' rows are quantised, coded, decoded, averaged and stepped by the two extra-gradient half-steps.
The products of the forward pass and of the gradients of activations are torch's.

    python examples/image_model.py --steps 300
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

    def __init__(self, vocabulary=12, width=32, heads=2, groups=4, side=6):
        self.n, self.D, self.H, self.G, self.side, self.P = vocabulary, width, heads, groups, side, side * side
        self.sizes = dict(norm_w=(width,), norm_b=(width,), wq=(width, width), bq=(width,), wk=(width, width), wv=(width, width), head=(width, vocabulary))
        self.at, self.d = {}, 0
        for name, shape in self.sizes.items():
            self.at[name] = self.d
            self.d += (math.prod(shape) + 3) // 4 * 4
        pairs = width // heads // 2
        self.rotary = qgx.Rotary.by_base((pairs - pairs // 2, pairs // 2), base=30.0)
        place = torch.arange(self.P, device="cuda")
        self.positions = torch.stack([place // side, place % side]).to(torch.int32)

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

    def gradients(self, ctx, X, V, embedding, tokens, targets, call):
        """tokens, targets [K, B, P].  Writes every run of V; returns the mean loss and what the backward pass worked from."""
        K, B, P, D, H = *tokens.shape, self.D, self.H
        p = {name: self.run_of(X, name) for name in self.sizes}
        x0 = embedding[tokens]                            # [K, B, P, D], channels last
        kept0 = ctx.new_checkpoint(x0.shape)              # tensor 0 of those that are kept in this call
        x, mean, rstd = ctx.group_norm(x0, self.G, p["norm_w"], p["norm_b"], activation="silu", keep=kept0, call_id=call)
        x = x.view(K, B * P, D)
        kept = ctx.checkpoint(x, call, tensor=1)

        def heads(t):                                     # [K, B P, D] -> [K, B, P, H, D / H]
            return t.view(K, B, P, H, D // H)

        def turn(t, back=False):
            return ctx.rotary(heads(t), self.rotary, self.positions, back=back)

        def flat(t):                                      # [K, B, H, P, D / H] -> [K, B P, D]
            return t.transpose(2, 3).reshape(K, B * P, D)

        q, k, v = (t.transpose(2, 3) for t in (turn(x @ p["wq"] + p["bq"]), turn(x @ p["wk"]), heads(x @ p["wv"])))
        scale = 1.0 / math.sqrt(D // H)
        attention = torch.softmax((q @ k.transpose(-1, -2)) * scale, -1)
        mixed = flat(attention @ v)
        kept_mixed = ctx.checkpoint(mixed, call, tensor=2)
        logits = mixed @ p["head"]
        logp = torch.log_softmax(logits, -1)
        seen = targets.view(K, B * P) >= 0
        t = targets.view(K, B * P).clamp_min(0)
        count = seen.sum(1).clamp_min(1).view(K, 1, 1)
        loss = -(logp.gather(2, t.unsqueeze(2)).squeeze(2) * seen).sum(1) / count.view(K)

        dlogits = (torch.exp(logp) - torch.nn.functional.one_hot(t, self.n)) * seen.unsqueeze(2) / count
        ctx.weight_gradient(kept_mixed, dlogits, self.run_of(V, "head"))
        dmixed = heads(dlogits @ p["head"].t()).transpose(2, 3)
        dattention = dmixed @ v.transpose(-1, -2)
        dv = flat(attention.transpose(-1, -2) @ dmixed)
        dscores = attention * (dattention - (attention * dattention).sum(-1, keepdim=True)) * scale
        dq, dk = (turn(flat(g), back=True).view(K, B * P, D) for g in (dscores @ k, dscores.transpose(-1, -2) @ q))
        ctx.weight_gradient(kept, dq, self.run_of(V, "wq"), db=self.run_of(V, "bq"))
        ctx.weight_gradient(kept, dk, self.run_of(V, "wk"))
        ctx.weight_gradient(kept, dv, self.run_of(V, "wv"))
        dx = dq @ p["wq"].t() + dk @ p["wk"].t() + dv @ p["wv"].t()
        ctx.group_norm_backward(dx.view(K, B, P, D), kept0, self.G, p["norm_w"], p["norm_b"], mean, rstd, "silu", dw=self.run_of(V, "norm_w"),
                                db=self.run_of(V, "norm_b"), need_dx=False)      # (the embedding is not learned)
        return loss.mean(), dict(kept0=kept0, kept=kept, kept_mixed=kept_mixed, dx=dx, dlogits=dlogits, dq=dq, dk=dk, dv=dv, mean=mean, rstd=rstd)


class Trainer:
    def __init__(self, K=4, batch=8, shift=(1, 2), max_norm=0.25, seed=0, model=None):
        self.model, self.K, self.batch, self.shift, self.max_norm = model or Model(), K, batch, shift, max_norm
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
        self.list = self.ctx.tensor_list([self.V])       # (the gradients are runs of V as they stand)
        self.calls = 0

    def data(self):
        m, (r, c) = self.model, self.shift
        tokens = torch.randint(0, m.n, (self.K, self.batch, m.side, m.side), generator=self.gen, device="cuda")
        targets = torch.full_like(tokens, -1)
        targets[..., :m.side - r, :m.side - c] = tokens[..., r:, c:]
        return tokens.flatten(-2), targets.flatten(-2)

    def dual_vectors(self, X, call):
        """The workers' clipped gradients at X in V, and their mean loss."""
        loss, _ = self.model.gradients(self.ctx, X, self.V, self.embedding, *self.data(), call)
        self.ctx.clip_gradients(self.list, self.max_norm, out=self.V)
        return loss

    def step(self):
        """One iteration: two rounds of gradients, coded exchange and half-step.  Returns the loss at its first point."""
        first, second = self.streams
        loss = self.dual_vectors(self.X, self.calls)
        self.ctx.quantize_encode(self.V, self.calls, first)
        self.ctx.eg_step(0, first, None, self.half)
        self.dual_vectors(self.half, self.calls + 1)
        self.ctx.quantize_encode(self.V, self.calls + 1, second)
        self.ctx.eg_step(1, second, first, self.X)
        self.calls += 2
        return loss


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=300)
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
