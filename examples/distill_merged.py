"""Retrains a merged head against the models it was merged from, then serves
it in 4 bits.

Several models had a head each; merged, one weight matrix serves them all.
What the unmerged heads answered is what the merged one should answer, so
their best classes teach it, with a low-rank adapter per model for what one
model needs for itself:

    log_probs         the teachers' best classes and their log probabilities
    adapt             every model's frames through the merged head and its adapter
    distill_backward  how far its logits are from the teachers' best, and the gradient
    adapt_backward    gradients of the weights, the bias and all adapters
    muon_step         orthogonalised momentum updates
    mx_quantize       the float32 weights as 4-bit ones
    mx_product        frames through them
    log_probs         and what they answer

    python examples/distill_merged.py [--models 3] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2201_07705_amd as P  # noqa: E402

TEMPERATURE = 2.0


def gradients(ctx, batch, x, weight, a, b, bias, indices, values):
    """Mean loss of a batch's rows against their teachers' best classes, and
    its gradients with respect to weight, bias and adapters."""
    logits = ctx.adapt(batch, x, weight, a, b, bias=bias)
    share = torch.full((len(x),), 1.0 / len(x), device="cuda")
    loss = torch.empty_like(share)
    dlogits = ctx.distill_backward(share, logits, indices, values, temperature=TEMPERATURE, loss=loss)
    grads = ctx.adapt_backward(batch, dlogits, x, weight, a, b, needs=("weight", "bias", "a", "b"))
    return loss, logits, dlogits, grads


def answers(ctx, weights, x, frames, top):
    """Best classes of each teacher's logits for its own frames."""
    best = [ctx.log_probs(part @ w.T, top=top) for part, w in zip(x.split(frames), weights)]
    return tuple(torch.cat([q[name] for q in best]) for name in ("top_indices", "top_log_probs"))


def run(models=3, n_in=256, classes=100, rank=4, frames=64, top=10, steps=60, lr=0.05, seed=0):
    """Returns the mean loss of every step; of the last frames, the share
    whose best class is the same in 4 bits as in bf16, and the mean loss of
    the 4-bit logits against the bf16 ones' best classes."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    ctx = P.Context(0, "bf16")
    try:
        common = normal(classes, n_in, std=2 * n_in ** -0.5)
        teachers = [(common + normal(classes, n_in, std=0.5 * n_in ** -0.5)).bfloat16() for _ in range(models)]
        # the merged head begins as the first model's
        master = {"weight": teachers[0].float(), "a": normal(models, rank, n_in, std=n_in ** -0.5),
                  "b": torch.zeros(models, classes, rank, device="cuda")}
        momentum = {k: torch.zeros_like(v) for k, v in master.items()}
        copy = {k: v.bfloat16() for k, v in master.items()}
        bias = torch.zeros(classes, device="cuda")
        batch = ctx.adapter_batch(range(models), [frames] * models, models, rank)
        losses = []
        for i in range(steps):
            x = normal(models * frames, n_in, std=1.0).bfloat16()
            indices, values = answers(ctx, teachers, x, frames, top)
            loss, _, _, grads = gradients(ctx, batch, x, copy["weight"], copy["a"], copy["b"], bias, indices, values)
            losses.append(loss.mean())
            for name, w in master.items():
                ctx.muon_step(w, momentum[name], grads[name], lr=lr * (1 - i / steps), copy=copy[name])
            bias -= lr * grads["bias"]
        # serving the merged weights: in bf16, and in 4 bits
        plain = ctx.adapter_batch([-1], [models * frames], 1, 1)
        wide = ctx.adapt(plain, x, copy["weight"], bias=bias)
        small = ctx.mx_product(x, ctx.mx_quantize(master["weight"]), bias=bias)
        best = ctx.log_probs(wide, top=top)
        same = best["top_indices"][:, 0] == ctx.log_probs(small, top=1)["top_indices"][:, 0]
        apart = ctx.distill(small, best["top_indices"], best["top_log_probs"])
        return [v.item() for v in losses], same.float().mean().item(), apart.mean().item()
    finally:
        ctx.close()


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--models", type=int, default=3)
    p.add_argument("--steps", type=int, default=60)
    args = p.parse_args()
    losses, same, apart = run(models=args.models, steps=args.steps)
    for i in sorted({0, *range(9, len(losses), 10), len(losses) - 1}):
        print(f"step {i + 1}: loss {losses[i]:.4f}")
    print(f"4 bits: {100 * same:.1f}% of the best classes are bf16's, loss against them {apart:.4f}")
