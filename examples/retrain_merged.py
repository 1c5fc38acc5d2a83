"""Retrains a merged projection with one low-rank adapter per model, then
serves single frames of all of them.

Several models share the weights of a layer. Merging costs each of them some
accuracy; what is lost is won back by training the shared weights on the
frames of all models together, with a small adapter for what one model needs
for itself. A step of that runs every operator of the framework's retraining
path:

    adapt            every model's frames through the shared weights and its adapter
    adapt_backward   gradients of the weights, the bias and all adapters
    muon_step        orthogonalised momentum updates of float32 weights, with
                     the bf16 copies that the next adapt reads

Here the layer has to learn a synthetic teacher: shared weights plus a
different low-rank part for each model.

    python examples/retrain_merged.py [--models 4] [--steps 80]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2201_07705_amd as P  # noqa: E402


class Layer:
    """float32 weights and momentum, and the bf16 copies that are computed with."""

    def __init__(self, ctx, models, n_in, n_out, rank, gen):
        def normal(*shape, std):
            return torch.randn(*shape, generator=gen, device="cuda") * std

        self.ctx = ctx
        self.master = {"weight": normal(n_out, n_in, std=n_in ** -0.5),
                       "a": normal(models, rank, n_in, std=n_in ** -0.5),
                       "b": torch.zeros(models, n_out, rank, device="cuda")}
        self.momentum = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.copy = {k: v.bfloat16() for k, v in self.master.items()}
        self.bias = torch.zeros(n_out, device="cuda")

    def __call__(self, batch, x):
        c = self.copy
        return self.ctx.adapt(batch, x, c["weight"], c["a"], c["b"], bias=self.bias)

    def step(self, batch, x, dy, lr):
        c = self.copy
        grads = self.ctx.adapt_backward(batch, dy, x, c["weight"], c["a"], c["b"],
                                        needs=("weight", "bias", "a", "b"))
        for name, w in self.master.items():
            self.ctx.muon_step(w, self.momentum[name], grads[name], lr=lr,
                               copy=c[name])
        # biases are vectors: a plain step
        self.bias -= lr * grads["bias"]


def teacher(models, n_in, n_out, rank, gen):
    """One weight matrix for each model: a shared one plus a low-rank part."""
    shared = torch.randn(n_out, n_in, generator=gen, device="cuda") * n_in ** -0.5
    left = torch.randn(models, n_out, rank, generator=gen, device="cuda") * n_out ** -0.5
    right = torch.randn(models, rank, n_in, generator=gen, device="cuda") * n_in ** -0.5
    return shared + left @ right


def run(models=4, n_in=256, n_out=96, rank=8, frames=64, steps=80, lr=0.05, seed=0):
    """Returns the loss of every step, and how far single served rows are
    from the same rows in a training batch (relative norm)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx = P.Context(0, "bf16")
    try:
        wanted = teacher(models, n_in, n_out, rank // 2, gen)
        layer = Layer(ctx, models, n_in, n_out, rank, gen)
        # the frames of every model are one stretch of rows
        batch = ctx.adapter_batch(range(models), [frames] * models, models, rank)
        losses = []
        for i in range(steps):
            x = torch.randn(models, frames, n_in, generator=gen, device="cuda").bfloat16()
            target = torch.bmm(x.float(), wanted.transpose(1, 2).contiguous())
            rows = x.view(-1, n_in)
            off = layer(batch, rows).float().view_as(target) - target
            losses.append(off.square().mean())
            dy = (off * (2.0 / (models * frames))).view(-1, n_out).bfloat16()
            layer.step(batch, rows, dy, lr * (1 - i / steps))
        y = layer(batch, rows)
        # serving: single frames in whatever order they arrive
        order = torch.randperm(models, generator=torch.Generator().manual_seed(seed)).tolist()
        picked = [m * frames + m % frames for m in order]
        single = ctx.adapter_batch(order, [1] * models, models, rank)
        served = layer(single, rows[picked])
        off = ((served.float() - y[picked].float()).norm() / y[picked].float().norm()).item()
        return [v.item() for v in losses], off
    finally:
        ctx.close()


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--models", type=int, default=4)
    p.add_argument("--steps", type=int, default=80)
    a = p.parse_args()
    losses, off = run(models=a.models, steps=a.steps)
    for i in sorted({0, *range(9, len(losses), 10), len(losses) - 1}):
        print(f"step {i + 1}: loss {losses[i]:.4f}")
    print(f"served rows differ from trained ones by {off:.1e} of their norm")
