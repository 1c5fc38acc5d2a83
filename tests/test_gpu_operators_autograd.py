"""What autograd is told of the operators, which it does not record."""

import pytest

from test_gpu_operators import batch_of, ctxs, problem  # noqa: F401

pytestmark = pytest.mark.gpu


def test_results_carry_no_graph(ctxs):  # noqa: F811
    ctx = ctxs["bf16"]
    s = problem("bf16", [5], [0], 1, 4, 32, 16)
    b = batch_of(ctx, s)
    for q in ("x", "w", "a", "b", "bias", "dy"):
        s[q].requires_grad_()
    y = ctx.adapt(b, s["x"], s["w"], s["a"], s["b"], bias=s["bias"])
    grads = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], s["a"], s["b"])
    for t in (y, ctx.orthogonalize(s["w"]), *grads.values()):
        assert not t.requires_grad and t.grad_fn is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_written_counts_as_changed(ctxs, dtype):  # noqa: F811
    """Every tensor passed to be written, and none that is only read."""
    import torch
    ctx = ctxs[dtype]
    s = problem(dtype, [5, 70], [0, 0], 1, 4, 32, 16)
    b = batch_of(ctx, s)
    args = (s["x"], s["w"], s["a"], s["b"])
    y = torch.empty(75, 16, dtype=s["x"].dtype, device="cuda")
    outputs = {k: torch.empty_like(v) for k, v in ctx.adapt_backward(b, s["dy"], *args).items()}
    o = torch.empty_like(s["w"])
    w, m, g = (torch.randn(24, 40, device="cuda") for _ in range(3))
    copy = w.bfloat16() if dtype == "bf16" else None
    read = [*args, s["dy"], s["bias"], g]
    written = [y, *outputs.values(), o, w, m] + ([copy] if dtype == "bf16" else [])
    before = {id(t): t._version for t in read + written}
    ctx.adapt(b, *args, bias=s["bias"], out=y)
    ctx.adapt_backward(b, s["dy"], *args, outputs=outputs)
    ctx.orthogonalize(s["w"], out=o)
    ctx.muon_step(w, m, g, lr=0.1, copy=copy)
    assert all(t._version == before[id(t)] for t in read)
    assert all(t._version > before[id(t)] for t in written)


def test_a_graph_that_saved_the_weights_is_refused(ctxs):  # noqa: F811
    import torch
    ctx = ctxs["bf16"]
    w, m, g = (torch.randn(24, 40, device="cuda") for _ in range(3))
    w.requires_grad_()
    loss = w.square().sum()
    ctx.muon_step(w, m, g, lr=0.1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    w.square().sum().backward()
    assert torch.equal(w.grad, 2 * w)


def test_inference_tensors(ctxs):  # noqa: F811
    import torch
    ctx = ctxs["f32"]
    with torch.inference_mode():
        w, m, g = (torch.randn(24, 40, device="cuda") for _ in range(3))
        before = w.clone()
        ctx.muon_step(w, m, g, lr=0.1)
        assert not torch.equal(w, before)
        ctx.orthogonalize(g, out=m)
