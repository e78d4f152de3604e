"""The plain forms that the layers' tests compare with, against independent values."""
import math

import numpy as np
import pytest
import torch

import layer_util as lu


def test_philox_known_answers():
    """The published known answers of Philox4x32-10."""
    def block(c, key):
        return [int(v) for v in lu.philox(np.array(c, dtype=object), key)]
    ones = 0xffffffff
    assert block([0, 0, 0, 0], 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert block([ones] * 4, ones << 32 | ones) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert block([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], 0x299f31d0 << 32 | 0xa4093822) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_mask_share_and_scale():
    m = lu.mask(400, 500, 0.25, 3, 9)
    assert set(m.unique().tolist()) == {0.0, 4 / 3}
    assert abs(float((m > 0).double().mean()) - 0.75) < 5 * math.sqrt(0.25 * 0.75 / 200000)


@pytest.mark.parametrize("name", [None, "relu", "gelu", "silu"])
def test_activations_and_slopes(name):
    z = torch.linspace(-6, 6, 1001, dtype=torch.float64)
    a, s, s2 = lu.act(name, z)
    torch_form = {None: lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
                  "silu": torch.nn.functional.silu}[name]
    assert torch.allclose(a, torch_form(z), atol=1e-14)
    h = 1e-5
    keep = z.abs() > 2 * h
    d = (lu.act(name, z + h)[0] - lu.act(name, z - h)[0]) / (2 * h)
    assert float((d - s)[keep].abs().max()) < 1e-9
    if name in ("gelu", "silu"):
        d = (lu.act(name, z + h)[1] - lu.act(name, z - h)[1]) / (2 * h)
        assert float(d.abs().max()) <= s2


def test_gradients_of_the_linear_layer():
    x, w, b = torch.randn(5, 7), torch.randn(3, 7), torch.randn(3)
    dy, keep = torch.randn(5, 3), lu.mask(5, 3, 0.5, 1, 2)
    leaves = [v.double().requires_grad_() for v in (x, w, b)]
    z = leaves[0] @ leaves[1].t() + leaves[2]
    y = torch.nn.functional.gelu(z) * keep
    ref, _, zz, dz = lu.linear(x, w, b, "gelu", keep, None, torch.float32)
    assert torch.allclose(ref, y.detach())
    want = torch.autograd.grad(y, leaves, dy.double())
    for (v, _), r in zip(lu.linear_grads(dy, x, w, zz, dz, "gelu", keep, torch.float32), want):
        assert torch.allclose(v, r)


def test_route_by_hand():
    inf = math.inf
    x = torch.tensor([[0.0, 2.0, 1.0, 2.0], [-inf, -inf, 3.0, -inf]])
    w, index, order, offsets, place = lu.route(x, 2, "softmax")
    assert index.tolist() == [[1, 3], [2, -1]] and w.tolist() == [[0.5, 0.5], [1.0, 0.0]]
    assert order.tolist() == [0, 2, 1, -1] and offsets.tolist() == [0, 0, 1, 2, 3]
    assert place.tolist() == [[0, 2], [1, -1]]
    # groups {0, 1} and {2, 3}: 0.6 + 0.1 against 0.5 + 0.3
    s = torch.tensor([[0.6, 0.1, 0.5, 0.3]])
    logits = torch.log(s / (1 - s))
    assert lu.route(logits, 1, "sigmoid", None, 2, 1)[1].tolist() == [[2]]
    assert lu.route(logits, 1, "sigmoid", torch.tensor([0.2, 0, 0, 0]), 2, 1)[1].tolist() == [[0]]
