"""Answers, distillation and 4-bit matrices without a GPU: every argument they
refuse is refused before the device is touched, with a status and a message,
and the binding's own checks raise."""

import ctypes

import pytest

from paper_2201_07705_amd import gemel as G

BIG = (1 << 32) + 1


@pytest.fixture
def ctx():
    c = G.Context(0, "bf16")
    yield c
    c.close()


def message(c):
    return c._lib.gemel_last_error(c._h).decode()


@pytest.mark.parametrize("change,why", [
    ({"rows": -1}, "rows must be"), ({"rows": (1 << 22) + 1}, "rows must be"),
    ({"classes": 0}, "classes must be"), ({"classes": (1 << 20) + 1}, "classes must be"),
    ({"dtype": 2}, "type of logits"), ({"t": 0.0}, "temperature"), ({"t": -1.0}, "temperature"),
    ({"t": float("nan")}, "temperature"), ({"t": float("inf")}, "temperature"), ({"t": 1e7}, "temperature"),
    ({"logits": None}, "logits is null"), ({"stride": 99}, "row stride"), ({"logits": 4097}, "aligned"),
    ({"k": 65}, "64"), ({"k": -1}, "64")])
def test_what_all_logits_calls_refuse(ctx, change, why):
    c = dict(rows=4, classes=100, logits=1 << 20, stride=100, dtype=0, k=5, t=1.0)
    c.update(change)
    a = G.Answers(entropy=4096, top_indices=8192)
    L, z = ctx._lib, (c["rows"], c["classes"], c["logits"], c["stride"], c["dtype"])
    calls = [lambda: L.gemel_log_probs(ctx._h, *z, None, c["k"], c["t"], a, None),
             lambda: L.gemel_distill(ctx._h, *z, 4096, 8192, c["k"], c["t"], 12288, None),
             lambda: L.gemel_distill_backward(ctx._h, z[0], z[1], None, *z[2:], 4096, 8192, c["k"], c["t"], 1 << 24, 100,
                                              None, None)]
    for call in calls:
        assert call() == G.EINVAL and why in message(ctx)


def test_log_probs_refusals(ctx):
    L = ctx._lib

    def call(labels=4096, top=3, out=G.Answers(entropy=8192), h=ctx._h):
        return L.gemel_log_probs(h, 4, 100, 1 << 20, 100, 0, labels, top, 1.0, out, None)

    assert call(h=None) == G.EINVAL
    for kw, why in [({"out": None}, "out is null"), ({"labels": None, "out": G.Answers(log_prob=8192)}, "labels is null"),
                    ({"labels": None, "out": G.Answers(rank=8192)}, "labels is null"), ({"out": G.Answers()}, "no output"),
                    ({"top": 0, "out": G.Answers(top_indices=8192)}, "no output"),
                    ({"out": G.Answers(entropy=8192, log_sum=8204)}, "overlaps"),
                    ({"out": G.Answers(entropy=4096)}, "overlaps"), ({"out": G.Answers(entropy=1 << 20)}, "overlaps")]:
        assert call(**kw) == G.EINVAL and why in message(ctx), kw
    # no rows: nothing to do, whatever the pointers are
    assert L.gemel_log_probs(ctx._h, 0, 100, None, 100, 0, None, 3, 1.0, G.Answers(), None) == G.OK
    assert L.gemel_distill(ctx._h, 0, 100, None, 100, 0, None, None, 3, 1.0, None, None) == G.OK


def test_distill_refusals(ctx):
    L = ctx._lib
    z = (1 << 20, 100, 0)
    for args, why in [((None, 8192, 3, 1.0, 12288), "indices is null"), ((4096, None, 3, 1.0, 12288), "values is null"),
                      ((4096, 8192, 0, 1.0, 12288), "entries"), ((4096, 8192, 3, 1.0, None), "loss is null"),
                      ((4096, 8192, 3, 1.0, 4100), "overlaps"), ((4096, 8192, 3, 1.0, 12289), "aligned")]:
        assert L.gemel_distill(ctx._h, 4, 100, *z, *args, None) == G.EINVAL and why in message(ctx), args
    back = [((4096, 8192, 3, 1.0, None, 100, None), "dlogits is null"), ((4096, 8192, 3, 1.0, 1 << 24, 99, None), "row stride"),
            ((4096, 8192, 3, 1.0, 1 << 20, 100, None), "overlaps"), ((4096, 8192, 3, 1.0, 1 << 24, 100, 1 << 24), "overlaps")]
    for args, why in back:
        assert L.gemel_distill_backward(ctx._h, 4, 100, None, *z, *args, None) == G.EINVAL and why in message(ctx), args


@pytest.mark.parametrize("q,why", [
    (None, "null"), (G.Mx(-1, 8, 4096, 8192), "rows"), (G.Mx(1 << 23, 8, 4096, 8192), "rows"), (G.Mx(4, 0, 4096, 8192), "columns"),
    (G.Mx(4, (1 << 20) + 1, 4096, 8192), "columns"), (G.Mx(4, 8, None, 8192), "null"), (G.Mx(4, 8, 4096, None), "null"),
    (G.Mx(4, 8, 4104, 8192), "16 bytes"), (G.Mx(4, 8, 4096, 8200), "16 bytes")])
def test_matrices_that_are_refused(ctx, q, why):
    L = ctx._lib
    for call in (lambda: L.gemel_mx_quantize(ctx._h, 1 << 20, 8, 0, q, None),
                 lambda: L.gemel_mx_dequantize(ctx._h, q, 1 << 20, 8, 0, None),
                 lambda: L.gemel_mx_product(ctx._h, 2, 1 << 20, 8, None, q, None, 1 << 21, 8, None)):
        assert call() == G.EINVAL and why in message(ctx)


def test_product_refusals(ctx):
    L, w = ctx._lib, G.Mx(16, 24, 4096, 1 << 16)
    x, y = 1 << 20, 1 << 21
    for args, why in [((2, x, 24, None, G.Mx(0, 24, None, None), None, y, 16), "no rows"), ((2, None, 24, None, w, None, y, 16), "either"),
                      ((-1, x, 24, None, w, None, y, 16), "rows must be"), ((2, x, 23, None, w, None, y, 16), "x has a bad"),
                      ((2, x, 24, None, w, None, None, 16), "y is null"), ((2, x, 24, None, w, None, y, 15), "y has a bad"),
                      ((2, x, 24, None, w, 4097, y, 16), "bias"), ((2, x, 24, None, w, None, x, 16), "overlaps"),
                      ((2, x, 24, None, w, None, 4096, 16), "overlaps"), ((2, None, 0, G.Mx(3, 24, 8192, 12288), w, None, y, 16), "xq"),
                      ((2, None, 0, G.Mx(2, 25, 8192, 12288), w, None, y, 16), "xq")]:
        assert L.gemel_mx_product(ctx._h, *args, None) == G.EINVAL and why in message(ctx), (args, message(ctx))
    assert L.gemel_mx_product(ctx._h, 0, None, 24, None, w, None, None, 16, None) == G.OK
    for dtype in (2, -1):
        assert L.gemel_mx_quantize(ctx._h, x, 24, dtype, w, None) == G.EINVAL and "type" in message(ctx)
        assert L.gemel_mx_dequantize(ctx._h, w, x, 24, dtype, None) == G.EINVAL and "type" in message(ctx)
    assert L.gemel_mx_quantize(ctx._h, 4096, 24, 0, w, None) == G.EINVAL and "overlaps" in message(ctx)


def test_binding_checks(ctx):
    torch = pytest.importorskip("torch")
    z, i = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="cuda"):
        ctx.log_probs(z, labels=i)
    with pytest.raises(ValueError, match="rows, classes"):
        ctx.log_probs(z[0])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ctx.log_probs(z.half())
    with pytest.raises(ValueError, match="rows, classes"):
        ctx.distill(z[0], i, z)
    with pytest.raises(ValueError, match="rows, cols"):
        ctx.mx_quantize(z[0])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ctx.mx_quantize(z.double())
    with pytest.raises(ValueError, match="cuda"):
        ctx.mx_quantize(z)
    with pytest.raises(ValueError, match="MxMatrix"):
        ctx.mx_product(z, z)
    codes, scales = G.MxMatrix.shapes(4, 600)
    assert codes == (4, 512) and scales == (2, 4, 16)
    q = G.MxMatrix(torch.zeros(codes, dtype=torch.uint8), torch.zeros(scales, dtype=torch.uint8), 4, 600)
    assert q.nbytes == 4 * 512 + 2 * 4 * 16
    with pytest.raises(ValueError, match="cuda"):
        ctx.mx_dequantize(q)


class Shape:
    """Stands for a tensor on the context's device of more elements than are
    there; the checks look at nothing else before they refuse it."""

    def __init__(self, *shape, dtype):
        import torch
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def new_empty(self, *a, **k):
        raise AssertionError("used")


def test_numbers_beyond_32_bits(ctx):
    torch = pytest.importorskip("torch")
    for shape in ((BIG, 1), (1, BIG)):
        z = Shape(*shape, dtype=torch.float32)
        for call in (lambda: ctx.log_probs(z), lambda: ctx.distill(z, z, z), lambda: ctx.distill_backward(None, z, z, z),
                     lambda: ctx.mx_quantize(z)):
            with pytest.raises(ValueError, match="32 bits"):
                call()
    z = Shape(4, 4, dtype=torch.float32)
    with pytest.raises(ValueError, match="top.* 32 bits"):
        ctx.log_probs(z, top=BIG)
    u8 = torch.uint8
    for rows, cols in ((BIG, 4), (4, BIG)):
        codes, scales = G.MxMatrix.shapes(rows, cols)
        q = G.MxMatrix(Shape(*codes, dtype=u8), Shape(*scales, dtype=u8), rows, cols)
        with pytest.raises(ValueError, match="32 bits"):
            ctx.mx_dequantize(q)
        with pytest.raises(ValueError, match="32 bits"):
            ctx.mx_product(z, q)


def test_a_description_is_made_again_where_the_matrix_is_another(ctx):
    torch = pytest.importorskip("torch")
    u8 = torch.uint8
    codes, scales = G.MxMatrix.shapes(4, 600)
    q = G.MxMatrix(Shape(*codes, dtype=u8), Shape(*scales, dtype=u8), 4, 600)
    first = ctx._mx("q", q)
    assert ctx._mx("q", q) is first and ctypes.sizeof(first) == 24
    q.codes = Shape(4, 511, dtype=u8)
    q.codes.data_ptr = lambda: 8192
    with pytest.raises(ValueError, match="codes must have shape"):
        ctx._mx("q", q)
    q.rows = 3
    with pytest.raises(ValueError, match="codes must have shape"):
        ctx._mx("q", q)
