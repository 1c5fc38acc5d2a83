"""Operands and results that share a matrix, and pointers that are not
aligned."""

import pytest

from test_gpu_operators import batch_of, close, ctxs, problem, reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1], [9, 30], [60, 70, 1]])
@pytest.mark.parametrize("k,n,gap", [(64, 48, 0), (33, 7, 1), (1000, 264, 3)])
def test_columns_of_one_matrix(ctxs, dtype, rows, k, n, gap):  # noqa: F811
    """Each result beside its operands in one wide matrix, whose other
    columns keep their values."""
    import torch
    from paper_2201_07705_amd import gemel as G
    ctx = ctxs[dtype]
    ids = [1, 0, -1][:len(rows)]
    s = problem(dtype, rows, ids, 2, 8, k, n, 51)
    want = reference(s)
    b = batch_of(ctx, s)
    m = sum(rows)
    wide = torch.full((m, 2 * (k + n) + 4 * gap), 7.0, dtype=s["x"].dtype, device="cuda")
    cut, at = {}, 0
    for name, width in (("y", n), ("x", k), ("dy", n), ("dx", k)):
        cut[name] = wide[:, at:at + width]
        at += width + gap
    cut["x"].copy_(s["x"])
    cut["dy"].copy_(s["dy"])
    ctx.adapt(b, cut["x"], s["w"], s["a"], s["b"], bias=s["bias"], out=cut["y"])
    got = ctx.adapt_backward(b, cut["dy"], cut["x"], s["w"], s["a"], s["b"], outputs={"x": cut["dx"]})
    close("y", cut["y"], want["y"])
    for name, t in got.items():
        close(name, t, want[name])
    assert torch.equal(cut["x"], s["x"]) and torch.equal(cut["dy"], s["dy"])
    kept = torch.ones(wide.shape[1], dtype=torch.bool)
    at = 0
    for width in (n, k, n, k):
        kept[at:at + width] = False
        at += width + gap
    assert bool((wide[:, kept.cuda()] == 7.0).all())
    # one column shared
    with pytest.raises(G.GemelError, match="overlaps"):
        ctx.adapt(b, wide[:, :k], s["w"], s["a"], s["b"], out=wide[:, k - 1:k - 1 + n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[9, 30], [60, 70]])
def test_shared_gradients_without_the_bank(ctxs, dtype, rows):  # noqa: F811
    s = problem(dtype, rows, [1, 0], 2, 8, 72, 40, 52)
    want = reference(s)
    ctx, b = ctxs[dtype], batch_of(ctxs[dtype], s)
    got = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], needs=("weight", "bias"))
    assert set(got) == {"weight", "bias"}
    for name, t in got.items():
        close(name, t, want[name])
