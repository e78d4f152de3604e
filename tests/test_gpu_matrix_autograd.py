"""What the matrix operators do where gradients are recorded (GPU)."""
import pytest

import paper_1607_00145_amd as g

pytestmark = pytest.mark.gpu


def test_a_gradient_is_refused_where_there_is_none(gpu):
    """Only mx_linear with a float weight has a gradient; what has none says so
    instead of returning a result without a graph."""
    import torch
    x = torch.randn(6, 64, device=gpu)
    xg = x.clone().requires_grad_()
    wq = g.mx_quantize(torch.randn(48, 64, device=gpu))
    xq = g.mx_quantize(x)
    C = torch.zeros(6, 48, device=gpu, requires_grad=True)
    O = torch.zeros(6, 64, device=gpu, requires_grad=True)
    calls = [lambda: g.mx_linear(xg, wq), lambda: g.mx_linear(xg.view(2, 3, 64), wq),
             lambda: g.mx_linear(xg * 2.0, wq), lambda: g.mx_matmul(xg, wq),
             lambda: g.mx_matmul(x, wq, C), lambda: g.mx_matmul(xq, wq, C, beta=1.0),
             lambda: g.orthogonalize(xg), lambda: g.orthogonalize(x, out=O),
             lambda: g.orthogonalize(xg.view(2, 3, 64)), lambda: xq.dequantize(out=O)]
    for i, call in enumerate(calls):
        with pytest.raises(RuntimeError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    assert (C != 0).any() and (O != 0).any()      # (written without recording)
    assert torch.equal(g.mx_linear(xg.detach(), wq), g.mx_matmul(x, wq))
    # a weight may be packed while it is trained: the packed copy is no tensor
    assert g.mx_quantize(xg).shape == (6, 64)
