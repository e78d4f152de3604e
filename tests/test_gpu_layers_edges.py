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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("e,groups", [(8, 1), (64, 4), (200, 1), (1000, 1)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_gradient_where_weights_are_nan(gpu, dtype, e, groups, scoring, renormalize):
    """A token whose weights are NaN has a gradient of NaN, whether or not what makes
    them so was chosen; the others' is theirs."""
    inf, k = math.inf, 3
    x = rand(e, 8, e, dtype=dtype)
    x[1, 3] = math.nan
    x[2, e - 1] = inf
    x[3] = -inf
    x[4] = math.nan
    x[5, ::2] = -inf
    x[6, ::2] = -inf
    x[6, 1] = math.nan
    bias = torch.zeros(e)
    bias[e - 1] = -5.0                      # (of the infinity's expert: not chosen)
    dw = rand(2, 8, k).to(gpu)
    how = dict(scoring=scoring, bias=bias.to(gpu), groups=groups, top_groups=max(1, groups // 2),
               renormalize=renormalize)
    leaf = x.to(gpu).requires_grad_()
    r = g.route(leaf, k, **how)
    dx, = torch.autograd.grad(r.weights, leaf, dw)
    nan = torch.tensor([False, True, scoring == "softmax", False, True, False, True, False], device=gpu)
    assert torch.equal(r.weights.isnan(), nan[:, None].expand(8, k))
    assert torch.equal(dx.isnan(), nan[:, None].expand(8, e))
    assert not dx[3].any()
    there = ~nan
    clean = x.to(gpu)[there].requires_grad_()
    want, = torch.autograd.grad(g.route(clean, k, **how).weights, clean, dw[there])
    assert torch.equal(dx[there], want)


# products --------------------------------------------------------------------

@pytest.mark.parametrize("dtype,m,n,k", [
    (torch.bfloat16, 1280, 2560, 256), (torch.float16, 2560, 1280, 256), (torch.bfloat16, 2560, 2560, 128),
    (torch.bfloat16, 2560, 768, 384), (torch.bfloat16, 1000, 2560, 320), (torch.float32, 640, 1280, 333),
    (torch.float32, 200, 4096, 200), (torch.bfloat16, 300, 300, 2000), (torch.float32, 1023, 515, 1000)])
def test_a_gradient_does_not_depend_on_what_else_is_wanted(gpu, dtype, m, n, k):
    """With w frozen dx is what it is beside dw, bit by bit, whatever tiles the products
    take and however many workgroups share their sums."""
    x, w, b = rand(1, m, k, dtype=dtype), rand(2, n, k, dtype=dtype, scale=k ** -0.5), rand(3, n, dtype=dtype)
    dy = rand(4, m, n, dtype=dtype).to(gpu)
    tensors = [v.to(gpu) for v in (x, w, b)]

    def gradients(*wanted):
        leaves = [t.detach().requires_grad_(i in wanted) for i, t in enumerate(tensors)]
        y = g.linear(*leaves, activation="silu")
        return torch.autograd.grad(y, [leaves[i] for i in wanted], dy)

    every = gradients(0, 1, 2)
    for wanted in ((0,), (1,), (2,), (0, 1), (0, 2), (1, 2)):
        for i, got in zip(wanted, gradients(*wanted)):
            assert torch.equal(got, every[i]), (wanted, i)


@pytest.mark.parametrize("p", [1e-6, 2.0 ** -17])
def test_a_probability_that_rounds_to_none(gpu, p):
    """It is p = 0: the same tensor comes back whatever the small number was."""
    x = rand(1, 20, 40).to(gpu)
    assert g.dropout(x, p, 5) is x and g.dropout(x, p, None) is x
    assert g.dropout(x, 2.0 ** -16, 5) is not x
    leaf = x.clone().requires_grad_()
    assert g.dropout(leaf, p, 5) is leaf
    w = rand(2, 30, 40).to(gpu)
    assert torch.equal(g.linear(x, w, activation="gelu", p=p, seed=3), g.linear(x, w, activation="gelu"))
