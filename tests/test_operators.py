"""The operators that serve and retrain merged layers, without a GPU: every
argument they refuse is refused before the device is touched, with a status
and a message, and the binding's own checks raise."""

import ctypes

import pytest

from paper_2201_07705_amd import gemel as G

I32 = ctypes.c_int32


def ints(*v):
    return (I32 * max(len(v), 1))(*v)


@pytest.fixture
def ctx():
    c = G.Context(0, "bf16")
    yield c
    c.close()


def message(c):
    return c._lib.gemel_last_error(c._h).decode()


@pytest.mark.parametrize("ids,rows,n,adapters,rank,ranks,scales,why", [
    ((0,), (1,), 1, 0, 8, None, None, "n_adapters"),
    ((0,), (1,), 1, 70000, 8, None, None, "n_adapters"),
    ((0,), (1,), 1, 2, 0, None, None, "max_rank"),
    ((0,), (1,), 1, 2, 257, None, None, "max_rank"),
    ((2,), (1,), 1, 2, 8, None, None, "unknown adapter"),
    ((-2,), (1,), 1, 2, 8, None, None, "unknown adapter"),
    ((0,), (-1,), 1, 2, 8, None, None, "negative row count"),
    ((0, 1), (1 << 21, 1 + (1 << 21)), 2, 2, 8, None, None, "at most"),
    ((0,), (1,), -1, 2, 8, None, None, "request arrays"),
    ((0,), (1,), 1, 2, 8, (8, 9), None, "rank must be"),
    ((0,), (1,), 1, 2, 8, (0, 8), None, "rank must be"),
    ((0,), (1,), 1, 2, 8, None, (1.0, float("nan")), "scale"),
    ((0,), (1,), 1, 2, 8, None, (float("inf"), 1.0), "scale"),
])
def test_batch_refusals(ctx, ids, rows, n, adapters, rank, ranks, scales, why):
    out = I32(7)
    st = ctx._lib.gemel_adapter_batch(
        ctx._h, ints(*ids), ints(*rows), n, adapters, rank,
        None if ranks is None else ints(*ranks),
        None if scales is None else (ctypes.c_float * len(scales))(*scales),
        ctypes.byref(out))
    assert st == G.EINVAL and why in message(ctx)
    assert out.value == 7


def test_null_arguments(ctx):
    L, out = ctx._lib, I32()
    assert L.gemel_adapter_batch(None, ints(0), ints(1), 1, 1, 1, None, None,
                                 ctypes.byref(out)) == G.EINVAL
    assert L.gemel_adapter_batch(ctx._h, ints(0), ints(1), 1, 1, 1, None,
                                 None, None) == G.EINVAL
    assert L.gemel_adapter_batch(ctx._h, None, ints(1), 1, 1, 1, None, None,
                                 ctypes.byref(out)) == G.EINVAL
    p = G.Projection(8, 8, 4096, 8, None, None, None)
    for b in (-1, 0, 3):
        assert L.gemel_adapt(ctx._h, b, ctypes.byref(p), 4096, 8, 8192, 8,
                             None) == G.EINVAL
        assert "unknown batch" in message(ctx)
        assert L.gemel_adapt_backward(ctx._h, b, ctypes.byref(p), 4096, 8,
                                      8192, 8, None, 0, None, None, None,
                                      None, None) == G.EINVAL
        assert L.gemel_adapter_batch_free(ctx._h, b) == G.EINVAL
    for f in (L.gemel_adapt,):
        assert f(None, 0, ctypes.byref(p), 4096, 8, 8192, 8, None) == G.EINVAL


@pytest.mark.parametrize("count,rows,cols,steps,g,out,why", [
    (-1, 4, 4, 5, 4096, 8192, "count"),
    (65536, 4, 4, 5, 4096, 8192, "count"),
    (1, 0, 4, 5, 4096, 8192, "rows and cols"),
    (1, 4, (1 << 20) + 1, 5, 4096, 8192, "rows and cols"),
    (1, 4, 4, 0, 4096, 8192, "steps"),
    (1, 4, 4, 17, 4096, 8192, "steps"),
    (1, 4, 4, 5, None, 8192, "g is null"),
    (1, 4, 4, 5, 4096, None, "out is null"),
    (1, 4, 4, 5, 4097, 8192, "aligned"),
    (1, 4, 4, 5, 4096, 4096 + 30, "overlaps"),
    (1, 4, 4, 5, 4096, 4096, "overlaps"),
])
def test_orthogonalize_refusals(ctx, count, rows, cols, steps, g, out, why):
    st = ctx._lib.gemel_orthogonalize(ctx._h, count, rows, cols, g, out, steps,
                                      None)
    assert st == G.EINVAL and why in message(ctx)


def test_muon_refusals(ctx):
    L = ctx._lib
    nan = float("nan")
    for args, why in [
        ((1, 4, 4, None, 8192, 12288, None, .1, .9, 0., 1, 5), "w is null"),
        ((1, 4, 4, 4096, None, 12288, None, .1, .9, 0., 1, 5), "momentum"),
        ((1, 4, 4, 4096, 8192, None, None, .1, .9, 0., 1, 5), "g is null"),
        ((1, 4, 4, 4096, 8192, 12288, None, nan, .9, 0., 1, 5), "finite"),
        ((1, 4, 4, 4096, 8192, 12288, None, .1, nan, 0., 1, 5), "finite"),
        ((1, 4, 4, 4096, 8192, 12288, None, .1, .9, nan, 1, 5), "finite"),
        ((1, 4, 4, 4096, 4096, 12288, None, .1, .9, 0., 1, 5), "overlaps"),
        ((1, 4, 4, 4096, 8192, 4100, None, .1, .9, 0., 1, 5), "overlaps"),
        ((1, 4, 4, 4096, 8192, 12288, 4096, .1, .9, 0., 1, 5), "overlaps"),
        ((1, 4, 4, 4098, 8192, 12288, None, .1, .9, 0., 1, 5), "aligned"),
        ((1, 4, 4, 4096, 8192, 12288, None, .1, .9, 0., 1, 0), "steps"),
    ]:
        assert L.gemel_muon_step(ctx._h, *args, None) == G.EINVAL
        assert why in message(ctx), (args, message(ctx))
    # nothing to do is not an error and touches no device
    assert L.gemel_muon_step(ctx._h, 0, 4, 4, None, None, None, None, .1, .9,
                             0., 1, 5, None) == G.OK
    c = G.Context(0, "f32")
    assert L.gemel_muon_step(c._h, 1, 4, 4, 4096, 8192, 12288, 16384, .1, .9,
                             0., 1, 5, None) == G.EINVAL
    assert "bf16 contexts" in c._lib.gemel_last_error(c._h).decode()
    c.close()


def test_binding_checks(ctx):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="length"):
        ctx.adapter_batch([0, 1], [1], 2, 8)
    with pytest.raises(ValueError, match="ranks"):
        ctx.adapter_batch([0], [1], 2, 8, ranks=[8])
    with pytest.raises(ValueError, match="scales"):
        ctx.adapter_batch([0], [1], 2, 8, scales=[1.0])
    with pytest.raises(G.GemelError) as e:
        ctx.adapter_batch([3], [1], 2, 8)
    assert e.value.code == G.EINVAL
    with pytest.raises(ValueError, match="cuda"):
        ctx.orthogonalize(torch.zeros(4, 4, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="rows, cols"):
        ctx.orthogonalize(torch.zeros(4, dtype=torch.bfloat16))
