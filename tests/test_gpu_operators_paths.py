"""Ways of working that the other tests' sizes do not reach: Newton-Schulz
steps that end on a whole pair, in batches; batches of several groups, the
last one shorter; and the thin products of float32 contexts held to float32.
Definitions and tolerances are those of the small cases: the relative norm of
the error of orthogonalised updates stays below 2^-8 in bf16 and 2^-17 in
float32, and beyond 5 steps grows with their number; whole numbers whose sums
stay below 2^24 are exact."""

import pytest

from test_gpu_operators import batch_of, ctxs, near, orthogonal, rand, DT  # noqa: F401
from test_gpu_operators_limits import whole

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2.0 ** -8, "f32": 2.0 ** -17}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [2, 3, 4, 6])
@pytest.mark.parametrize("rows,cols", [(512, 4608), (4608, 512), (300, 3001)])
def test_orthogonalize_in_pairs(ctxs, dtype, steps, rows, cols):  # noqa: F811
    import torch
    gen = torch.Generator(device="cuda").manual_seed(steps)
    g = rand(gen, 2, rows, cols, dtype=DT[dtype])
    g[1] *= 2.0 ** 10
    got = ctxs[dtype].orthogonalize(g, steps=steps)
    for q, o in zip(g, got):
        near(o, orthogonal(q, steps), TOL[dtype] * max(1.0, steps / 2.5))


def step(ctx, dtype, w, m, g, steps):
    """muon_step against its definition, matrix by matrix."""
    import torch
    f64 = torch.float64
    copy = torch.empty_like(w, dtype=torch.bfloat16) if dtype == "bf16" else None
    w0, m0 = w.clone(), m.clone()
    ctx.muon_step(w, m, g, lr=0.3, momentum=0.9, weight_decay=0.1, steps=steps, copy=copy)
    rate = 0.3 * max(1.0, w.shape[1] / w.shape[2]) ** 0.5
    for i in range(w.shape[0]):
        m1 = 0.9 * m0[i].to(f64) + g[i].to(f64)
        o = orthogonal(g[i].to(f64) + 0.9 * m1, steps)
        assert ((m[i].to(f64) - m1).abs() <= 2.0 ** -22 * (1.9 * m1.abs() + g[i].abs())).all(), i
        off = w[i].to(f64) - ((1 - 0.3 * 0.1) * w0[i].to(f64) - rate * o)
        assert off.norm() <= rate * 2.0 ** -17 * max(1.0, steps / 2.5) * o.norm() + 2.0 ** -22 * w0[i].norm(), i
    if copy is not None:
        assert torch.equal(copy, w.bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [2, 4, 5])
@pytest.mark.parametrize("rows,cols", [(512, 4608), (4608, 512)])
def test_muon_step_in_pairs(ctxs, dtype, steps, rows, cols):  # noqa: F811
    import torch
    gen = torch.Generator(device="cuda").manual_seed(steps)
    w, m, g = (rand(gen, 2, rows, cols, std=s, dtype=torch.float32) for s in (1.0, 1e-2, 1e-2))
    step(ctxs[dtype], dtype, w, m, g, steps)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count,rows,cols", [(130, 1024, 1000), (440, 300, 2000)])
def test_batches_of_several_groups(ctxs, dtype, count, rows, cols):  # noqa: F811
    """Planes of all matrices would take more than 4 GiB."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(count)
    g = rand(gen, count, rows, cols, dtype=DT[dtype])
    g *= (torch.arange(count, device="cuda") % 7 + 1).view(-1, 1, 1)
    got = ctxs[dtype].orthogonalize(g, steps=2)
    for q, o in zip(g, got):
        near(o, orthogonal(q, 2), TOL[dtype])
    w, m, u = (rand(gen, count, rows, cols, std=s, dtype=torch.float32) for s in (1.0, 1e-2, 1e-2))
    step(ctxs[dtype], dtype, w, m, u, 2)


@pytest.mark.parametrize("n_rows", [[3, 9], [50, 70]])
@pytest.mark.parametrize("ranks", [[3, 2], [2, 1]])
def test_thin_products_of_float32_keep_their_bits(ctxs, n_rows, ranks):  # noqa: F811
    """Sums x A^T of up to 2^20, which 16 bits would not hold."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(sum(n_rows))
    f32, f64 = torch.float32, torch.float64
    m, k, n, rank = sum(n_rows), 4, 4, 3
    x, a = whole(gen, m, k, top=127, dtype=f32) * 4 + 1, whole(gen, 2, rank, k, top=127, dtype=f32) * 4 + 1
    dy, b = whole(gen, m, n, top=127, dtype=f32) * 4 + 1, whole(gen, 2, n, rank, top=127, dtype=f32) * 4 + 1
    w, one, row = torch.zeros(n, k, device="cuda"), whole(gen, 2, n, rank, top=1, dtype=f32), whole(gen, 2, rank, k, top=1, dtype=f32)
    ctx, s = ctxs["f32"], dict(ids=[1, 0], n_rows=n_rows, bank=2, rank=rank, ranks=ranks, scales=[1.0, -2.0])
    batch = batch_of(ctx, s)
    y = ctx.adapt(batch, x, w, a, one)
    dx = ctx.adapt_backward(batch, dy, x, w, row, b, needs=("x",))["x"]
    at = 0
    for rows, i in zip(n_rows, s["ids"]):
        q, r = slice(at, at + rows), ranks[i]
        t = s["scales"][i] * x[q].to(f64) @ a[i, :r].T.to(f64)
        assert t.abs().max() > 2 ** 17
        assert torch.equal(y[q].to(f64), t @ one[i, :, :r].T.to(f64))
        u = s["scales"][i] * dy[q].to(f64) @ b[i, :, :r].to(f64)
        assert torch.equal(dx[q].to(f64), u @ row[i, :r].to(f64))
        at += rows
