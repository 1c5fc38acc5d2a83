"""Tensors that a caller passes for answers which a call does not give are
refused, not left as they were. No GPU is needed."""

import pytest

from paper_2201_07705_amd import gemel as G
from test_answers import Shape

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("outputs,labels,top,why", [
    ({"log_probs": 1}, True, 3, "log_probs"), ({"entropy": 1, "ranks": 1}, True, 3, "ranks"), ({"rank": 1}, False, 3, "rank"),
    ({"log_prob": 1}, False, 0, "log_prob"), ({"top_indices": 1}, True, 0, "top_indices")])
@pytest.mark.parametrize("needs", [None, ("entropy",)])
def test_names_that_are_no_answers(outputs, labels, top, why, needs):
    ctx = G.Context(0, "bf16")
    z, i = Shape(4, 10, dtype=torch.float32), Shape(4, dtype=torch.int32)
    with pytest.raises(ValueError, match=f"outputs: no answer '{why}'"):
        ctx.log_probs(z, labels=i if labels else None, top=top, needs=needs, outputs=outputs)
    ctx.close()
