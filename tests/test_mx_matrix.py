"""The tensors of a 4-bit matrix are looked at again whenever they are other
ones, or were changed in place, wherever they lie. No GPU is needed."""

import pytest

from paper_2201_07705_amd import gemel as G
from test_answers import Shape

torch = pytest.importorskip("torch")
U8 = torch.uint8


@pytest.fixture
def ctx():
    c = G.Context(0, "bf16")
    yield c
    c.close()


def matrix(ctx):
    codes, scales = G.MxMatrix.shapes(4, 600)
    q = G.MxMatrix(Shape(*codes, dtype=U8), Shape(*scales, dtype=U8), 4, 600)
    assert ctx._mx("q", q) is ctx._mx("q", q)   # (checked once, and used)
    return q


class Strided(Shape):
    def is_contiguous(self):
        return False


class Elsewhere(Shape):
    def get_device(self):
        return -1


@pytest.mark.parametrize("name,right", [("codes", (4, 512)), ("scales", (2, 4, 16))])
def test_other_tensors_at_the_same_address(ctx, name, right):
    for other, why in ((Shape(*right[:-1], right[-1] - 1, dtype=U8), "shape"), (Shape(1, *right[1:], dtype=U8), "shape"),
                       (Shape(*right, dtype=torch.int16), "uint8"), (Strided(*right, dtype=U8), "contiguous"),
                       (Elsewhere(*right, dtype=U8), "cuda:0")):
        q = matrix(ctx)
        setattr(q, name, other)
        with pytest.raises(ValueError, match=f"{name}.*{why}"):
            ctx._mx("q", q)
        with pytest.raises(ValueError, match=f"{name}.*{why}"):
            ctx._mx("q", q)
        setattr(q, name, Shape(*right, dtype=U8))
        ctx._mx("q", q)


@pytest.mark.parametrize("name", ["codes", "scales"])
def test_tensors_that_are_changed_in_place(ctx, name):
    q = matrix(ctx)
    t = getattr(q, name)
    t.shape = torch.Size((1, *t.shape[1:]))
    if name == "scales":
        t.shape = torch.Size((1, 4, 16))
    with pytest.raises(ValueError, match=f"{name}.*shape"):
        ctx._mx("q", q)
    q = matrix(ctx)
    getattr(q, name).is_contiguous = lambda: False
    with pytest.raises(ValueError, match=f"{name}.*contiguous"):
        ctx._mx("q", q)


def test_other_sizes(ctx):
    for name, value in (("rows", 5), ("cols", 1025)):
        q = matrix(ctx)
        setattr(q, name, value)
        with pytest.raises(ValueError, match="codes.*shape"):
            ctx._mx("q", q)
