"""The operators at the ends of their ranges. Where inputs are small whole
numbers every partial sum is one too, below 2^24 and so exact in float32:
results then have to be equal to the definition's, whatever the order."""

import pytest

from test_gpu_operators import batch_of, ctxs, DT  # noqa: F401

pytestmark = pytest.mark.gpu


def whole(gen, *shape, top, dtype):
    """Whole numbers from -top to top."""
    import torch
    return torch.randint(-top, top + 1, shape, generator=gen, device="cuda",
                         dtype=torch.int8).to(dtype)


def whole_problem(dtype, n_rows, ids, bank, rank, k, n, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, m = DT[dtype], sum(n_rows)
    return dict(x=whole(gen, m, k, top=2, dtype=dt), w=whole(gen, n, k, top=1, dtype=dt),
                a=whole(gen, bank, rank, k, top=1, dtype=dt),
                b=whole(gen, bank, n, rank, top=1, dtype=dt),
                bias=whole(gen, n, top=3, dtype=torch.float32), dy=whole(gen, m, n, top=1, dtype=dt),
                n_rows=n_rows, ids=ids, bank=bank, rank=rank, ranks=[rank] * bank,
                scales=[1.0] * bank, k=k, n=n, m=m, dtype=dtype)


def definition(s):
    """y and the gradients in 64 bits, a stretch of rows at a time."""
    import torch
    f64 = torch.float64
    w, a, b = (s[q].to(f64) for q in ("w", "a", "b"))
    y, dx = torch.empty(s["m"], s["n"], device="cuda"), torch.empty(s["m"], s["k"], device="cuda")
    out = {"weight": torch.zeros_like(w), "bias": torch.zeros_like(s["bias"], dtype=f64),
           "a": torch.zeros_like(a), "b": torch.zeros_like(b)}
    at = 0
    for count, i in zip(s["n_rows"], s["ids"]):
        for p in range(at, at + count, 1 << 18):
            q = slice(p, min(at + count, p + (1 << 18)))
            x, dy = s["x"][q].to(f64), s["dy"][q].to(f64)
            t, u = x @ a[i].T, dy @ b[i]
            y[q] = (x @ w.T + s["bias"] + t @ b[i].T).float()
            dx[q] = (dy @ w + u @ a[i]).float()
            out["weight"] += dy.T.contiguous() @ x
            out["bias"] += dy.sum(0)
            out["a"][i] += u.T.contiguous() @ x
            out["b"][i] += dy.T.contiguous() @ t
        at += count
    return dict(out, y=y, x=dx)


@pytest.mark.parametrize("k,n", [(16, 65), (140, 70)])
def test_more_rows_than_a_transposed_copy_holds(ctxs, k, n):  # noqa: F811
    """float32 gradients of 2^21 + 1 rows, which the host once accepted and
    then failed half-way."""
    import torch
    rows = (1 << 21) + 1
    s = whole_problem("f32", [rows - 77, 77], [1, 0], 2, 3, k, n, 5)
    want = definition(s)
    ctx, b = ctxs["f32"], batch_of(ctxs["f32"], s)
    got = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], s["a"], s["b"])
    got["y"] = ctx.adapt(b, s["x"], s["w"], s["a"], s["b"], bias=s["bias"])
    for name, t in got.items():
        assert torch.equal(t.double(), want[name].double()), name


def test_more_tiles_than_a_grid_of_the_smallest(ctxs):  # noqa: F811
    """2^22 rows of 8256 outputs (69 GB)."""
    import torch
    rows, n, k = 1 << 22, 8256, 8
    s = whole_problem("bf16", [rows - 9, 9], [-1, 0], 1, 2, k, n, 6)
    ctx, b = ctxs["bf16"], batch_of(ctxs["bf16"], s)
    del s["dy"]
    y = ctx.adapt(b, s["x"], s["w"], s["a"], s["b"], bias=s["bias"])
    f64 = torch.float64
    x, w = s["x"].to(f64), s["w"].to(f64)
    for q in (slice(0, 300), slice(rows // 2 - 5, rows // 2 + 5), slice(rows - 300, rows)):
        want = x[q] @ w.T + s["bias"]
        if q.stop == rows:
            want[-9:] += x[-9:] @ s["a"][0].to(f64).T @ s["b"][0].to(f64).T
        assert torch.equal(y[q], want.to(torch.bfloat16))
    # every row was written: whole numbers, their sums over the outputs
    assert torch.equal(y.view(1024, -1, n)[:, 0].sum(1, dtype=torch.float32),
                       (x.view(1024, -1, k)[:, 0] @ w.T + s["bias"]).to(torch.bfloat16).sum(1, dtype=torch.float32))


@pytest.mark.parametrize("small", [2.0 ** -10, 2.0 ** -20, 2.0 ** -24, 2.0 ** -30])
def test_values_far_below_the_largest_of_their_row(ctxs, small):  # noqa: F811
    """float32 gradients of one large row of dy among small ones, for inputs
    that the large row has at zero: each operand is off by 2^-22 of itself or
    2^-38 of the largest one that it is multiplied beside, a product by
    2^-22, and a sum of 2048 by as many roundings of 2^-24."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    m, k, n = 2048, 256, 80
    x = torch.randn(m, k, generator=gen, device="cuda")
    dy = torch.randn(m, n, generator=gen, device="cuda") * small
    dy[77] /= small
    x[77, :128] = 0
    w = torch.randn(n, k, generator=gen, device="cuda")
    ctx = ctxs["f32"]
    b = ctx.adapter_batch([-1], [m], 1, 1)
    got = ctx.adapt_backward(b, dy, x, w, needs=("weight", "x"))
    f64 = torch.float64

    def off(t, axis):
        t = t.to(f64).abs()
        return torch.maximum(2.0 ** -22 * t, 2.0 ** -38 * t.amax(axis, keepdim=True))

    dyd, xd, wd = dy.to(f64), x.to(f64), w.to(f64)
    for name, p, q, ep, eq in (
            ("weight", dyd.T, xd, off(dy, 0).T, off(x, 0)), ("x", dyd, wd, off(dy, 1), off(w, 0))):
        mag = p.abs() @ q.abs()
        bound = ep @ q.abs() + p.abs() @ eq + ep @ eq + (2.0 ** -22 + 2.0 ** -24 * (p.shape[1] + 8)) * mag
        assert ((got[name].to(f64) - p.contiguous() @ q).abs() <= bound).all(), name
