"""Products of more bf16 values than 2^30 with 4-bit weights: the last rows of
aligned ones, and of ones that are copied piece by piece, are those of the
same rows alone, within what another order of sums may change."""

import pytest

from paper_2201_07705_amd import gemel as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pad", [0, 1])
def test_more_values_than_are_copied_at_once(pad):
    import torch
    ctx = G.Context(0, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(9)
    rows, k, n = (1 << 20) + 300, 1048, 24
    x = torch.empty(rows, k + pad, device="cuda", dtype=torch.bfloat16)[:, pad:]
    x[:] = torch.randn(k, device="cuda", generator=gen)
    # (around the pieces' ends too: 2^30 values are 1024512 rows)
    some = torch.cat([torch.arange(40, device="cuda"), 1024512 + torch.arange(-20, 20, device="cuda"), torch.arange(rows - 40, rows, device="cuda")])
    x[some] = torch.randn(len(some), k, device="cuda", generator=gen).bfloat16()
    w = ctx.mx_quantize(torch.randn(n, k, device="cuda", generator=gen))
    bias = torch.randn(n, device="cuda", generator=gen)
    y = ctx.mx_product(x, w, bias=bias)
    left, right = x[some].double(), ctx.mx_dequantize(w, dtype=torch.float32).double()
    want, size = left @ right.T + bias.double(), left.abs() @ right.abs().T + bias.double().abs()
    # (k / 4 + 70 additions follow each other at most, 2^-24 of the magnitudes each; half a step of bf16 for y)
    tol = size * (k / 4 + 70) * 2.0 ** -24
    assert ((y[some].double() - want).abs() <= tol + (want.abs() + tol) * 2.0 ** -8).all()
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[some] = False
    same = y[others]
    assert torch.equal(same, same[:1].expand_as(same))
    ctx.close()
