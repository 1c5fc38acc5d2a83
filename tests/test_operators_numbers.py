"""Numbers beyond 32 bits: the C interface takes int32, to which ctypes cuts
whatever it is given without a word, so the binding refuses them. No GPU is
needed."""

import pytest

from paper_2201_07705_amd import gemel as G

BIG = (1 << 32) + 1


@pytest.fixture
def ctx():
    c = G.Context(0, "bf16")
    yield c
    c.close()


@pytest.mark.parametrize("args,kw,why", [
    (([1 << 32], [1], 2, 8), {}, "adapter_ids"),
    (([-(1 << 32)], [1], 2, 8), {}, "adapter_ids"),
    (([0], [BIG], 2, 8), {}, "n_rows"),
    (([0], [1], BIG, 8), {}, "n_adapters"),
    (([0], [1], 2, (1 << 32) + 8), {}, "rank"),
    (([0], [1], 2, 8), {"ranks": [8, BIG]}, "ranks"),
])
def test_batches(ctx, args, kw, why):
    with pytest.raises(ValueError, match=why + ".* 32 bits"):
        ctx.adapter_batch(*args, **kw)


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
        raise AssertionError("used")

    new_empty = stride = data_ptr


def test_shapes_and_steps(ctx):
    torch = pytest.importorskip("torch")
    for shape in ((BIG, 1), (1, BIG), (BIG, 1, 1)):
        with pytest.raises(ValueError, match="32 bits"):
            ctx.orthogonalize(Shape(*shape, dtype=torch.bfloat16))
        t = Shape(*shape, dtype=torch.float32)
        with pytest.raises(ValueError, match="32 bits"):
            ctx.muon_step(t, t, t, lr=0.1)
    g = Shape(4, 4, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="steps.* 32 bits"):
        ctx.orthogonalize(g, steps=BIG + 4)
    t = Shape(4, 4, dtype=torch.float32)
    with pytest.raises(ValueError, match="steps.* 32 bits"):
        ctx.muon_step(t, t, t, lr=0.1, steps=BIG + 4)
    batch = G.AdapterBatch(ctx, 0, 1, 1, 8)
    for shape in ((BIG, 4), (4, BIG)):
        with pytest.raises(ValueError, match="32 bits"):
            ctx.adapt(batch, None, Shape(*shape, dtype=torch.bfloat16))
