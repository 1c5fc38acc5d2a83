"""Answers, distillation, gradients, updates and 4-bit products together, as a
user runs them: the example runs, its gradients are those of the formulas in
64 bits, and the 4-bit head answers as its weights say."""

import math
import os
import sys

import pytest

from paper_2201_07705_amd import gemel as G

pytestmark = pytest.mark.gpu


@pytest.fixture
def example():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    import distill_merged
    yield distill_merged
    sys.path.remove(os.path.join(root, "examples"))


@pytest.mark.parametrize("models,n_in,classes,frames,top", [(3, 256, 100, 64, 10), (2, 130, 1003, 5, 20), (1, 33, 17, 1, 17)])
def test_the_example_runs(example, models, n_in, classes, frames, top):
    losses, same, apart = example.run(models=models, n_in=n_in, classes=classes, frames=frames, top=top, steps=6)
    assert len(losses) == 6 and all(math.isfinite(v) and v > -1e-4 for v in losses)
    assert 0 <= same <= 1 and math.isfinite(apart)


def test_its_gradients(example):
    """Against the formulas in 64 bits from the same bf16 logits: dlogits is
    off by its rounding to bf16 (eps / 2, 2^-8 of each) and 2000 of 2^-24 of dloss T
    (p + q); sums of the gradients by that times the other factor, and by
    float32 additions (2^-24 for each of at most 200 in a row, and bf16 pairs
    of the thin products, 2^-15)."""
    import torch
    ctx = G.Context(0, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    models, frames, k, n, r, t = 3, 40, 96, 70, 4, example.TEMPERATURE
    rows = models * frames
    x, w = normal(rows, k).bfloat16(), normal(n, k, std=2 * k ** -0.5).bfloat16()
    a, b = normal(models, r, k, std=k ** -0.5).bfloat16(), normal(models, n, r, std=0.3).bfloat16()
    bias = normal(n)
    teachers = [normal(n, k, std=2 * k ** -0.5).bfloat16() for _ in range(models)]
    indices, values = example.answers(ctx, teachers, x, frames, 9)
    batch = ctx.adapter_batch(range(models), [frames] * models, models, r)
    loss, logits, dlogits, grads = example.gradients(ctx, batch, x, w, a, b, bias, indices, values)
    p = (logits.double() / t).softmax(1)
    q = torch.zeros_like(p).scatter_add(1, indices.long(), (values.double() / t).softmax(1))
    g = t / rows * (p - q)
    g_tol = g.abs() * 2.0 ** -8 + t / rows * (p + q) * 2000 * 2.0 ** -24
    assert ((dlogits.double() - g).abs() <= g_tol).all()
    lp = (logits.double() / t).log_softmax(1)
    lq = (values.double() / t).log_softmax(1)
    want = t * t * (lq.exp() * (lq - lp.gather(1, indices.long()))).sum(1)
    assert ((loss.double() - want).abs() <= 4 * 2000 * 2.0 ** -24 * (1 + want)).all()

    def near(got, left, right, left_tol):
        exact, size = left.T @ right, left.abs().T @ right.abs()
        tol = left_tol.T @ right.abs() + size * (200 * 2.0 ** -24 + 2.0 ** -15)
        assert ((got.double() - exact).abs() <= tol).all()

    xd = x.double()
    near(grads["weight"], g, xd, g_tol)
    assert ((grads["bias"].double() - g.sum(0)).abs() <= g_tol.sum(0) + 200 * 2.0 ** -24 * g.abs().sum(0)).all()
    for m in range(models):
        mine = slice(m * frames, (m + 1) * frames)
        ad, bd = a[m].double(), b[m].double()
        near(grads["b"][m], g[mine], xd[mine] @ ad.T, g_tol[mine])
        low, low_tol = g[mine] @ bd, g_tol[mine] @ bd.abs() + g[mine].abs() @ bd.abs() * (100 * 2.0 ** -24)
        near(grads["a"][m], low, xd[mine], low_tol)
    ctx.close()


def test_four_bits_answer_as_their_values_say(example):
    """The 4-bit head's answers are those of a bf16 head that holds its values
    (which bf16 does exactly): logits rounded once to bf16 in both."""
    import torch
    ctx = G.Context(0, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn(1003, 512, generator=gen, device="cuda") * 0.1
    q = ctx.mx_quantize(w)
    for rows in (1, 33, 1100):
        x = torch.randn(rows, 512, generator=gen, device="cuda").bfloat16()
        y = ctx.mx_product(x, q)
        plain = ctx.adapter_batch([-1], [rows], 1, 1)
        z = ctx.adapt(plain, x, ctx.mx_dequantize(q))
        size = x.double().abs() @ ctx.mx_dequantize(q, dtype=torch.float32).double().abs().T
        # Two sums in orders of their own, each then rounded by at most half a
        # step (2^-8 of it): |y - z| <= |y - s| + |s - t| + |t - z|, where the
        # sums s and t are at most (1 + 2^-8) times as large as y and z.
        sums = size * 400 * 2.0 ** -24
        half = 2.0 ** -8 * (1 + 2.0 ** -8)
        assert ((y.double() - z.double()).abs() <= (y.double().abs() + z.double().abs()) * half + sums).all()
        best = ctx.log_probs(y, top=3)
        labels = best["top_indices"][:, 1].contiguous()
        again = ctx.log_probs(y, labels=labels)
        assert (again["rank"] == 1).all()
        assert torch.equal(again["log_prob"], best["top_log_probs"][:, 1])
        # a model is not apart from itself
        loss = ctx.distill(y, *(ctx.log_probs(y, top=64)[k] for k in ("top_indices", "top_log_probs")))
        mass = ctx.log_probs(y, top=64)["top_log_probs"].double().exp().sum(1)
        assert ((loss.double() + mass.log()).abs() <= 2000 * 2.0 ** -24).all()
    ctx.close()
