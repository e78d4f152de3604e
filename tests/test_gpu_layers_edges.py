"""The layers' operators at the edges of what they say: gradients of numbers that are
none, one gradient without the others, results in place of an operand, probabilities
that round to none, masks in 16 bits."""
import math

import pytest
import torch

import layer_util as lu
import paper_1607_00145_amd as g
from test_gpu_layers import rand
from test_gpu_layers_more import CODES, TYPES, on_gpu
from test_layers_abi import product_tiles

pytestmark = pytest.mark.gpu


# routing ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("e", [1, 8, 200, 1000])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_gradient_of_a_token_without_experts(gpu, dtype, e, scoring, renormalize):
    """It is zero, and the others' is theirs."""
    x, k = rand(e, 6, e, dtype=dtype), min(e, 3)
    x[::2] = -math.inf
    dw = rand(2, 6, k).to(gpu)
    leaf, clean = x.to(gpu).requires_grad_(), x[1::2].to(gpu).requires_grad_()
    how = dict(scoring=scoring, renormalize=renormalize)
    dx, = torch.autograd.grad(g.route(leaf, k, **how).weights, leaf, dw)
    want, = torch.autograd.grad(g.route(clean, k, **how).weights, clean, dw[1::2])
    assert bool((dx[::2] == 0).all()) and torch.equal(dx[1::2], want)
