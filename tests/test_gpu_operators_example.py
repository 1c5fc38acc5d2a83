"""The retraining example: the operators together, as a user runs them."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def example():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    import retrain_merged
    yield retrain_merged
    sys.path.remove(os.path.join(root, "examples"))


@pytest.mark.parametrize("models,n_in,n_out", [(4, 256, 96), (3, 130, 45)])
def test_the_merged_layer_learns(example, models, n_in, n_out):
    losses, off = example.run(models=models, n_in=n_in, n_out=n_out, steps=80)
    assert len(losses) == 80
    # a random layer misses a random teacher by twice the targets' size (and
    # the adapters' part); after training most of that is gone
    assert losses[0] > 1.0
    assert sum(losses[-5:]) / 5 < 0.1 * losses[0]
    # the same rows in another batch: both results are rounded once to bf16
    assert off <= 2.0 ** -8
