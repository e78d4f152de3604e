"""Orthogonalised stacks of matrices: memory layouts (GPU)."""
import pytest

import paper_1607_00145_amd as g

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,rows,cols", [(12, 256, 64), (5, 33, 47), (3, 300, 200), (2, 70, 700)])
def test_interleaved_stacks(gpu, heads, rows, cols, dtype):
    """The heads of a weight [rows, heads, cols], and of its transpose: matrices
    whose rows lie between those of the others."""
    import torch
    t = getattr(torch, dtype)
    guard = torch.randn(rows, heads * cols + 9, device=gpu).to(t)
    W = guard[:, 4:4 + heads * cols]
    G = W.view(rows, heads, cols).transpose(0, 1)
    want = g.orthogonalize(G.contiguous())
    assert torch.equal(g.orthogonalize(G), want)
    out = torch.full_like(guard, 3.0)
    O = out[:, 4:4 + heads * cols].view(rows, heads, cols).transpose(0, 1)
    assert g.orthogonalize(G, out=O) is O
    assert torch.equal(O, want)
    assert (out[:, :4] == 3.0).all() and (out[:, -5:] == 3.0).all()
    before = guard.clone()
    assert g.orthogonalize(G, out=G) is G
    assert torch.equal(G, want)
    assert torch.equal(guard[:, :4], before[:, :4]) and torch.equal(guard[:, -5:], before[:, -5:])
    wide = before[:, 4:4 + heads * cols].t().contiguous()      # [heads * cols, rows]
    T = wide.view(heads, cols, rows).transpose(1, 2)
    assert torch.equal(g.orthogonalize(T, out=T), want)


def test_overlapping_stacks_are_refused(gpu):
    import torch
    buf = torch.randn(4096, device=gpu)
    for shape, stride in (((2, 8, 64), (32, 64, 1)), ((3, 8, 8), (60, 8, 1)), ((2, 5, 6), (6, 6, 1))):
        O = buf.as_strided(shape, stride)
        with pytest.raises(g.GettError):
            g.orthogonalize(torch.randn(shape, device=gpu), out=O)


@pytest.mark.parametrize("shape", [(0, 5, 7), (3, 0, 7), (3, 5, 0), (2, 3, 0, 5), (2, 3, 5, 0),
                                   (2, 0, 4, 5), (0, 0, 4, 5)])
def test_empty_stacks(gpu, shape):
    import torch
    G = torch.randn(shape, device=gpu)
    assert g.orthogonalize(G).shape == shape
    assert g.orthogonalize(G, out=G) is G
    strided = torch.randn(*shape[:-1], 2 * shape[-1] + 1, device=gpu)[..., :2 * shape[-1]:2]
    assert g.orthogonalize(strided).shape == shape


@pytest.mark.parametrize("shape", [(2, 3, 0), (2, 0, 8), (0, 3, 8), (2, 0, 0), (0,)])
def test_linear_of_empty_leading_dimensions(gpu, shape):
    """As for two dimensions: a sum over nothing is zero."""
    import torch
    x = torch.randn(shape, device=gpu)
    w = torch.randn(6, shape[-1], device=gpu)
    for y in (g.mx_linear(x, w), g.mx_linear(x, g.mx_quantize(w))):
        assert y.shape == (*shape[:-1], 6) and (y == 0).all()
    x.requires_grad_()
    w.requires_grad_()
    g.mx_linear(x, w).sum().backward()
    assert x.grad.shape == x.shape and (w.grad == 0).all()


def test_linear_of_a_vector(gpu):
    import torch
    x, w = torch.randn(64, device=gpu), torch.randn(48, 64, device=gpu)
    assert torch.equal(g.mx_linear(x, w), g.mx_linear(x[None], w)[0])
    with pytest.raises(ValueError):
        g.mx_linear(x[0], w)
