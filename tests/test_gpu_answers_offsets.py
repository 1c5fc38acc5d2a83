"""Answers, gradients and 4-bit matrices whose elements lie beyond 2^32: the
last rows are those of the same rows alone."""

import pytest

from paper_2201_07705_amd import gemel as G

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctxs():
    c = {d: G.Context(0, d) for d in ("bf16", "f32")}
    yield c
    for q in c.values():
        q.close()


def wide(rows, cols, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.empty(rows, cols, dtype=dtype, device="cuda")
    x[:] = torch.randn(cols, device="cuda", generator=gen)
    x[-40:] = torch.randn(40, cols, device="cuda", generator=gen) * 3
    return x


@pytest.mark.parametrize("rows,cols", [(36000, 120001), (9000000 // 2, 1000)])
def test_logits(ctxs, rows, cols):
    import torch
    if rows > 1 << 22:
        rows = 1 << 22
    ctx = ctxs["bf16"]
    z = wide(rows, cols + 100, torch.bfloat16)[:, :cols]
    assert z.stride(0) * (rows - 40) > 2 ** 32 - 2 ** 28
    labels = torch.arange(rows, device="cuda", dtype=torch.int32) % cols
    whole = ctx.log_probs(z, labels=labels, top=7)
    index, value = whole["top_indices"], whole["top_log_probs"]
    alone = ctx.log_probs(z[-40:], labels=labels[-40:], top=7)
    for name in whole:
        assert torch.equal(whole[name][-40:], alone[name]), name
    value = torch.roll(value, 1, dims=1).contiguous()
    loss = torch.empty(rows, device="cuda")
    grad = ctx.distill_backward(None, z, index, value, loss=loss)
    few = torch.empty(40, device="cuda")
    last = ctx.distill_backward(None, z[-40:], index[-40:], value[-40:], loss=few)
    assert torch.equal(grad[-40:], last) and torch.equal(loss[-40:], few)
    assert torch.equal(ctx.distill(z, index, value)[-40:], few)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matrices(ctxs, dtype):
    import torch
    ctx = ctxs[dtype]
    rows, cols = 70000, 65600
    x = wide(rows, cols, torch.bfloat16 if dtype == "bf16" else torch.float32)
    q = ctx.mx_quantize(x)
    last = ctx.mx_quantize(x[-40:])
    assert torch.equal(q.codes[-40:], last.codes) and torch.equal(q.scales[:, -40:], last.scales)
    v = ctx.mx_dequantize(q)
    assert torch.equal(v[-40:], ctx.mx_dequantize(last)) and torch.equal(v[:1], ctx.mx_dequantize(ctx.mx_quantize(x[:1])))
    del v
    w = ctx.mx_quantize(wide(130, cols, torch.float32) / 100)
    eps = torch.finfo(x.dtype).eps / 2
    for left, few in ((q, last), (x, x[-40:])):
        y = ctx.mx_product(left, w)
        z = ctx.mx_product(few, w).double()
        # (other paths sum in another order: 2^-24 for each of cols / 4 + 70 additions)
        a, b = (ctx.mx_dequantize(few, dtype=torch.float32) if left is q else few).double(), ctx.mx_dequantize(w, dtype=torch.float32).double()
        tol = (a.abs() @ b.abs().T) * 2 * (cols / 4 + 70) * 2.0 ** -24 + 2 * eps * z.abs()
        assert ((y[-40:].double() - z).abs() <= tol).all()
        # weights of as many rows: outputs of the others
        t = ctx.mx_product(ctx.mx_quantize(wide(130, cols, torch.float32) / 100) if left is q else w_values(ctx, w, x.dtype), q)
        assert ((t[:, -40:].double().T - a_times(ctx, last, b)).abs() <= (a_values(ctx, last).abs() @ b.abs().T) *
                (cols / 4 + 70) * 2.0 ** -24 + eps * t[:, -40:].double().T.abs() + 1e-30).all()
        del y, t


def a_values(ctx, q):
    import torch
    return ctx.mx_dequantize(q, dtype=torch.float32).double()


def a_times(ctx, q, b):
    return a_values(ctx, q) @ b.T


def w_values(ctx, w, dtype):
    return ctx.mx_dequantize(w, dtype=dtype)
