"""The example: a network trained with 4-bit products and orthogonalised
updates, and served from packed weights."""
import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_training_and_serving(gpu):
    import torch

    import paper_1607_00145_amd as g
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import mx_training as example
    finally:
        sys.path.pop(0)
    weights, x, losses = example.train(steps=40)
    assert losses[-1] < 0.5 * losses[0], losses
    packed = [g.mx_quantize(w) for w in weights]
    many = example.forward(x, weights)
    # the same roundings; sums of at most 256 products in another order can
    # move a hidden value across a rounding step (a sixth of it) now and then
    for i in (0, 100, 511):
        one = example.forward(x[i:i + 1], packed)
        assert torch.allclose(one, many[i:i + 1], atol=0.05 * float(many.abs().max()))
