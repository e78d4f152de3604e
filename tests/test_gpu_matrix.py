"""The matrix operators on the GPU against plain 64-bit forms (matrix_util).

Tolerances, from the operators' arithmetic:
- packing is exact: equal values.
- a product's sum of k terms in 32 bits: (k + 2) u sum |a b|, u = 2^-24 (any
  order of summation), and half a unit in the last place of the result's type.
- an orthogonalised matrix, relative to its norm: each of the three products
  of a step rounds its operands to 2^-22 (two parts) and the step's map
  magnifies what it is given by at most 4 (its derivative on [0, 1.2]):
  12 steps 2^-22; for bf16 (one part, 2^-12) the fifteen roundings are
  independent and add in squares: 4 sqrt(3 steps) 2^-12; and the result's own
  rounding."""
import math

import numpy as np
import pytest

import paper_1607_00145_amd as g
from matrix_util import mx_values, newton_schulz

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]
HALF_ULP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # eps / 2
MUON = (3.4445, -4.7750, 2.0315)


def torch_type(name):
    import torch
    return getattr(torch, name)


def matrix(rng, rows, cols, dtype, kind="dense", scale=1.0):
    """A device matrix with values of many sizes, laid out as `kind` says."""
    import torch
    v = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (1, cols))) * scale
    t = torch.from_numpy(v).to(torch_type(dtype)).cuda()
    if kind == "dense":
        return t
    if kind == "transposed":
        return t.t().contiguous().t()
    if kind == "slice":                       # odd pitch, unaligned start
        w = torch.full((rows, cols + 13), 7.0, dtype=t.dtype, device=t.device)
        w[:, 5:5 + cols] = t
        return w[:, 5:5 + cols]
    if kind == "strided":                     # no direction is stride-one
        w = torch.full((rows, 2 * cols), 7.0, dtype=t.dtype, device=t.device)
        w[:, ::2] = t
        return w[:, ::2]
    raise ValueError(kind)


def host(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------ quantisation ---

SHAPES = [(1, 1), (1, 31), (1, 33), (2, 256), (5, 257), (16, 128), (33, 100), (127, 129),
          (130, 300), (257, 513), (1, 4096), (300, 64), (129, 1)]


@pytest.mark.parametrize("kind", ["dense", "transposed", "slice", "strided"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_values(gpu, rows, cols, dtype, kind):
    import torch
    rng = np.random.default_rng(rows * 1000 + cols)
    x = matrix(rng, rows, cols, dtype, kind)
    want, want_t = mx_values(host(x)), mx_values(host(x).T)
    q, qt = g.mx_quantize(x, "both")
    assert q.shape == (rows, cols) and qt.shape == (cols, rows)
    for p, w in ((q, want), (qt, want_t), (g.mx_quantize(x), want),
                 (g.mx_quantize(x, "rows"), want_t)):
        assert np.array_equal(host(p.dequantize()), w)
        # values with their scale are numbers of bfloat16
        assert np.array_equal(host(p.dequantize(torch.bfloat16)), w)


@pytest.mark.parametrize("along", ["cols", "rows", "both"])
def test_quantize_one_and_both_give_the_same_bytes(gpu, along):
    rng = np.random.default_rng(5)
    x = matrix(rng, 200, 300, "float32")
    q, qt = g.mx_quantize(x, "both")
    one = {"cols": (g.mx_quantize(x), q), "rows": (g.mx_quantize(x, "rows"), qt),
           "both": (g.mx_quantize(x.t(), "rows"), q)}[along]
    assert (one[0].codes == one[1].codes).all()
    rows = 200 if one[0].rows == 200 else 300
    R = (rows + 15) // 16 * 16
    view = lambda p: p.scales.view(-1, R, 4)[:, :rows]      # of rows past the last: anything
    assert (view(one[0]) == view(one[1])).all()


def test_quantize_special_values(gpu):
    import torch
    x = torch.zeros(8, 96)
    x[0, 3] = math.inf
    x[1, 40] = -math.inf
    x[2, 70] = math.nan
    x[3, :32] = 1e-40                       # a block below the smallest scale
    x[3, 32] = 2.0 ** -126
    x[4, :] = 3.0e38
    x[4, 1] = -1.0
    x[5, ::2] = -0.0
    x[6, :7] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])   # ties, scale 1
    x[6, 7] = 7.9                           # beyond the largest: becomes 6
    x[7, :4] = torch.tensor([1.0, 0.999999, 2.0 ** -30, -4.000001])
    for dev in (x.cuda(), x.t().contiguous().t().cuda()):
        got = host(g.mx_quantize(dev).dequantize())
        assert np.array_equal(got, mx_values(x.numpy()), equal_nan=True)
        got = host(g.mx_quantize(dev, "rows").dequantize())
        assert np.array_equal(got, mx_values(x.numpy().T), equal_nan=True)
    assert np.isnan(got).sum() == 3 * 8


def test_quantize_leaves_neighbours_alone(gpu):
    """Outputs in a guarded buffer: nothing outside gett_mx_size's bytes."""
    import torch
    for rows, cols in ((1, 1), (17, 257), (130, 250)):
        x = torch.randn(rows, cols, device="cuda")
        sizes = g.gett_mx_size(rows, cols)[1:] + g.gett_mx_size(cols, rows)[1:]
        gap = 256
        buf = torch.full((sum(sizes) + 5 * gap,), 0xA5, dtype=torch.uint8, device="cuda")
        at, p = [], gap
        for n in sizes:
            at.append(p)
            p += n + gap
        base = buf.data_ptr()
        st = g.gett_mx_quantize(0, rows, cols, x.data_ptr(), cols, 1, *[base + a for a in at],
                                torch.cuda.current_stream().cuda_stream)
        assert st == 0
        keep = torch.ones_like(buf, dtype=torch.bool)
        for a, n in zip(at, sizes):
            keep[a:a + n] = False
        assert (buf[keep] == 0xA5).all()


@pytest.mark.parametrize("kind", ["dense", "transposed", "slice", "strided"])
def test_dequantize_into_strided_memory(gpu, kind):
    import torch
    rng = np.random.default_rng(7)
    x = matrix(rng, 70, 290, "float32")
    want = mx_values(host(x))
    out = matrix(rng, 70, 290, "float32", kind)
    whole = out._base if out._base is not None else out
    before = whole.clone()
    g.mx_quantize(x).dequantize(out=out)
    assert np.array_equal(host(out), want)
    if kind in ("slice", "strided"):
        out.copy_(torch.as_strided(before, out.shape, out.stride(), out.storage_offset()))
        assert (whole == before).all()


def test_empty_matrices(gpu):
    import torch
    for shape in ((0, 5), (5, 0), (0, 0)):
        q = g.mx_quantize(torch.zeros(shape, device="cuda"))
        assert q.dequantize().shape == shape
    a = g.mx_quantize(torch.zeros(3, 0, device="cuda"))
    b = g.mx_quantize(torch.zeros(4, 0, device="cuda"))
    assert (g.mx_matmul(a, b) == 0).all()
    C = torch.full((3, 4), 2.0, device="cuda")
    assert (g.mx_matmul(a, b, C, beta=0.5) == 1.0).all()
    assert (g.mx_matmul(torch.zeros(3, 0, device="cuda"), b, C, beta=0.5) == 0.5).all()


# ---------------------------------------------------------------- products ---

def product_close(got, a, b, dtype, alpha=1.0, beta=0.0, C=None):
    """got against alpha a b^T + beta C in 64 bits; a, b are the values."""
    ref = alpha * (a @ b.T) + (beta * C if beta else 0.0)
    size = abs(alpha) * (np.abs(a) @ np.abs(b).T) + (np.abs(beta * C) if beta else 0.0)
    bound = (a.shape[1] + 2) * 2.0 ** -24 * size + HALF_ULP[dtype] * np.abs(ref) * 1.01
    if dtype == "float16":
        bound = bound + 2.0 ** -24
    err = np.abs(got - ref)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), float((err / np.maximum(bound, 1e-300)).max())


PRODUCTS = [(1, 1, 1), (1, 5, 33), (2, 64, 256), (3, 40, 300), (15, 33, 1000), (16, 31, 255),
            (17, 100, 512), (31, 65, 2100), (32, 32, 32), (33, 33, 700), (64, 64, 64),
            (65, 127, 513), (128, 130, 1024), (100, 300, 257), (260, 259, 300), (7, 2000, 5000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(gpu, m, n, k, dtype):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    x, w = matrix(rng, m, k, dtype, scale=0.1), matrix(rng, n, k, dtype, scale=0.1)
    a, b = mx_values(host(x)), mx_values(host(w))
    wq = g.mx_quantize(w)
    packed = g.mx_matmul(g.mx_quantize(x), wq, dtype=x.dtype)
    assert packed.dtype == x.dtype
    product_close(host(packed), a, b, dtype)
    product_close(host(g.mx_matmul(x, wq)), a, b, dtype)      # quantised in the call


# (tiles of every size, and rows that end inside one)
@pytest.mark.parametrize("m,n,k", [(4100, 4097, 300), (2049, 2050, 260), (1500, 2600, 512)])
def test_product_large_tiles(gpu, m, n, k):
    rng = np.random.default_rng(m)
    x, w = matrix(rng, m, k, "bfloat16"), matrix(rng, n, k, "bfloat16")
    a, b = mx_values(host(x)), mx_values(host(w))
    product_close(host(g.mx_matmul(x, g.mx_quantize(w), dtype=torch_type("float32"))), a, b,
                  "float32")


@pytest.mark.parametrize("kind", ["dense", "transposed", "slice", "strided"])
@pytest.mark.parametrize("m,n,k", [(1, 70, 300), (20, 50, 600), (90, 140, 500), (300, 40, 260),
                                   (40, 7, 300)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_product_accumulates_into_any_layout(gpu, m, n, k, kind, dtype):
    import torch
    rng = np.random.default_rng(m + n + k)
    x, w = matrix(rng, m, k, dtype, "slice", 0.1), matrix(rng, n, k, dtype, scale=0.1)
    a, b = mx_values(host(x)), mx_values(host(w))
    wq = g.mx_quantize(w)
    for left in (g.mx_quantize(x), x):
        C = matrix(rng, m, n, dtype, kind)
        whole = C._base if C._base is not None else C
        before, C0 = whole.clone(), host(C)
        assert g.mx_matmul(left, wq, C, alpha=0.75, beta=-0.5) is C
        product_close(host(C), a, b, dtype, 0.75, -0.5, C0)
        if kind in ("slice", "strided"):
            C.copy_(torch.as_strided(before, C.shape, C.stride(), C.storage_offset()))
            assert (whole == before).all()


def test_product_beta_zero_does_not_read_c(gpu):
    import torch
    x, w = torch.randn(40, 64, device="cuda"), torch.randn(50, 64, device="cuda")
    wq = g.mx_quantize(w)
    C = torch.full((40, 50), math.nan, device="cuda")
    assert torch.isfinite(g.mx_matmul(x, wq, C)).all()
    C.fill_(2.0)
    x.fill_(math.nan)                       # alpha 0: A is not read
    assert (g.mx_matmul(x, wq, C, alpha=0.0, beta=3.0) == 6.0).all()


@pytest.mark.parametrize("m", [1, 5, 20, 100, 300])
def test_product_of_nan_blocks(gpu, m):
    """A block with an infinity makes its row's results NaN, no others."""
    import torch
    x, w = torch.randn(m, 600, device="cuda"), torch.randn(77, 600, device="cuda")
    x[m // 2, 599] = math.inf
    w[13, 300] = math.nan
    y = g.mx_matmul(x, g.mx_quantize(w))
    bad = torch.zeros(m, 77, dtype=torch.bool, device="cuda")
    bad[m // 2] = True
    bad[:, 13] = True
    assert (torch.isnan(y) == bad).all()
    y = g.mx_matmul(g.mx_quantize(x), g.mx_quantize(w))
    assert (torch.isnan(y) == bad).all()


def test_product_repeats_bit_for_bit(gpu):
    import torch
    for m, n, k in ((1, 512, 4096), (24, 512, 4096), (128, 128, 8192), (300, 700, 1000)):
        x, w = torch.randn(m, k, device="cuda"), g.mx_quantize(torch.randn(n, k, device="cuda"))
        first = g.mx_matmul(x, w)
        for _ in range(3):
            assert torch.equal(g.mx_matmul(x, w), first)


# ------------------------------------------------------------ linear layer ---

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 40, 64), (33, 65, 100), (130, 70, 257)])
def test_linear_gradients(gpu, m, n, k, dtype):
    rng = np.random.default_rng(m)
    x, w = matrix(rng, m, k, dtype, scale=0.1), matrix(rng, n, k, dtype, scale=0.1)
    dy = matrix(rng, m, n, dtype, scale=0.1)
    x.requires_grad_()
    w.requires_grad_()
    y = g.mx_linear(x, w)
    y.backward(dy)
    X, W, DY = host(x.detach()), host(w.detach()), host(dy)
    product_close(host(y.detach()), mx_values(X), mx_values(W), dtype)
    product_close(host(x.grad), mx_values(DY), mx_values(W.T), dtype)
    product_close(host(w.grad), mx_values(DY.T), mx_values(X.T), dtype)


def test_linear_gradient_against_differences(gpu):
    """Where all values are numbers of the 4-bit grid the rounding does
    nothing, and the gradients are those of x w^T: the differences of a
    function that is linear in each argument, exact."""
    import torch
    rng = np.random.default_rng(3)
    # each block of 32 holds a 4: scale 1 along both directions
    def grid(rows, cols):
        v = rng.choice([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0], (rows, cols))
        v[::16] = 4.0
        v[:, ::16] = 4.0
        return torch.from_numpy(v).float().cuda()
    x, w, dy = grid(64, 96), grid(32, 96), grid(64, 32)
    x.requires_grad_()
    w.requires_grad_()
    (g.mx_linear(x, w) * dy).sum().backward()
    f = lambda a, b: ((host(a) @ host(b).T) * host(dy)).sum()
    for t, other, first in ((x.detach(), w.detach(), True), (w.detach(), x.detach(), False)):
        grad = x.grad if first else w.grad
        for i, j in ((0, 0), (3, 17), (31, 95)):
            up, down = t.clone(), t.clone()
            up[i, j] += 0.5
            down[i, j] -= 0.5
            d = f(up, other) - f(down, other) if first else f(other, up) - f(other, down)
            assert d == float(grad[i, j])


def test_linear_broadcast_gradient_and_leading_dimensions(gpu):
    import torch
    x = torch.randn(2, 3, 64, device="cuda", requires_grad=True)
    w = torch.randn(48, 64, device="cuda", requires_grad=True)
    y = g.mx_linear(x, w)
    assert y.shape == (2, 3, 48)
    y.sum().backward()                       # the gradient has zero strides
    ones = np.ones((6, 48))
    product_close(host(x.grad).reshape(6, 64), ones, mx_values(host(w.detach()).T), "float32")
    product_close(host(w.grad), ones.T, mx_values(host(x.detach()).reshape(6, 64).T), "float32")


def test_linear_needs_only_what_it_is_asked_for(gpu):
    import torch
    x, w = torch.randn(40, 64, device="cuda"), torch.randn(48, 64, device="cuda")
    plain = g.mx_linear(x, w)
    assert torch.equal(plain, g.mx_linear(x, g.mx_quantize(w)))
    for a, b in ((True, False), (False, True)):
        xa, wb = x.clone().requires_grad_(a), w.clone().requires_grad_(b)
        y = g.mx_linear(xa, wb)
        assert torch.equal(y.detach(), plain)
        y.backward(torch.ones_like(y))
        assert (xa.grad is not None) == a and (wb.grad is not None) == b


def test_linear_of_two_types_and_layouts(gpu):
    """x, w and dy in layouts and types of their own; the gradients come in
    the types of what they are the gradients of."""
    rng = np.random.default_rng(12)
    for tx, tw, kx, kw, ky in (("bfloat16", "float32", "transposed", "slice", "dense"),
                               ("float16", "bfloat16", "strided", "transposed", "transposed"),
                               ("float32", "float32", "slice", "dense", "strided")):
        x, w = matrix(rng, 150, 90, tx, kx, 0.1), matrix(rng, 70, 90, tw, kw, 0.1)
        dy = matrix(rng, 150, 70, tx, ky, 0.1)
        x.requires_grad_()
        w.requires_grad_()
        y = g.mx_linear(x, w)
        y.backward(dy)
        assert x.grad.dtype == x.dtype and w.grad.dtype == w.dtype
        X, W, DY = host(x.detach()), host(w.detach()), host(dy)
        product_close(host(y.detach()), mx_values(X), mx_values(W), tx)
        product_close(host(x.grad), mx_values(DY), mx_values(W.T), tx)
        product_close(host(w.grad), mx_values(DY.T), mx_values(X.T), tw)


def test_linear_into_given_memory(gpu):
    """gett_mx_linear and its gradient into column-major results (the products
    exchange their operands)."""
    import torch
    rng = np.random.default_rng(13)
    m, n, k = 140, 200, 260
    x, w, dy = (matrix(rng, *s, "float32", scale=0.1) for s in ((m, k), (n, k), (m, n)))
    (c1, s1), (c2, s2) = g.gett_mx_size(k, m)[1:], g.gett_mx_size(k, n)[1:]
    parts = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (c1, s1, c2, s2)]
    p = [t.data_ptr() for t in parts]
    y, dx, dw = (torch.empty(c, r, device="cuda").t() for r, c in ((m, n), (m, k), (n, k)))
    stream = torch.cuda.current_stream().cuda_stream
    assert g.gett_mx_linear(m, n, k, 0, x.data_ptr(), k, 1, 0, w.data_ptr(), k, 1, y.data_ptr(), 1,
                            m, *p, stream) == 0
    assert g.gett_mx_linear_grad(m, n, k, 0, dy.data_ptr(), n, 1, *p, dx.data_ptr(), 1, m, 0,
                                 dw.data_ptr(), 1, n, stream) == 0
    X, W, DY = host(x), host(w), host(dy)
    product_close(host(y), mx_values(X), mx_values(W), "float32")
    product_close(host(dx), mx_values(DY), mx_values(W.T), "float32")
    product_close(host(dw), mx_values(DY.T), mx_values(X.T), "float32")


@pytest.mark.parametrize("m,n,k", [(0, 5, 7), (5, 0, 7), (5, 7, 0)])
def test_linear_of_empty_matrices(gpu, m, n, k):
    import torch
    x = torch.randn(m, k, device="cuda", requires_grad=True)
    w = torch.randn(n, k, device="cuda", requires_grad=True)
    y = g.mx_linear(x, w)
    assert y.shape == (m, n) and (y == 0).all()
    y.backward(torch.ones_like(y))
    assert (x.grad == 0).all() and (w.grad == 0).all()


@pytest.mark.parametrize("m,n,k", [(2000, 300, 280), (3000, 40, 600), (20, 3000, 30)])
def test_linear_steps_of_uneven_sizes(gpu, m, n, k):
    """The gradients' two products take tiles of different sizes, or one of
    them none."""
    rng = np.random.default_rng(m)
    x, w, dy = (matrix(rng, *s, "bfloat16", scale=0.1) for s in ((m, k), (n, k), (m, n)))
    x.requires_grad_()
    w.requires_grad_()
    y = g.mx_linear(x, w)
    y.backward(dy)
    X, W, DY = host(x.detach()), host(w.detach()), host(dy)
    product_close(host(y.detach()), mx_values(X), mx_values(W), "bfloat16")
    product_close(host(x.grad), mx_values(DY), mx_values(W.T), "bfloat16")
    product_close(host(w.grad), mx_values(DY.T), mx_values(X.T), "bfloat16")


# -------------------------------------------------------- orthogonalisation ---

def orth_tolerance(dtype, steps):
    if dtype == "bfloat16":
        return 4 * math.sqrt(3 * max(steps, 1)) * 2.0 ** -12 + HALF_ULP[dtype]
    return 12 * max(steps, 1) * 2.0 ** -22 + HALF_ULP[dtype]


def stack(rng, shape, dtype, scale=1e-3):
    import torch
    r, c = shape[-2:]
    k = max(1, min(r, c) // 16)
    v = rng.standard_normal((*shape[:-2], r, k)) @ rng.standard_normal((*shape[:-2], k, c))
    v = v / math.sqrt(k) + rng.standard_normal(shape)
    return torch.from_numpy(v * scale).to(torch_type(dtype)).cuda()


def orth_close(got, G, dtype, steps=5, poly=MUON, eps=1e-7):
    ref = newton_schulz(host(G), steps, poly, eps)
    got = host(got)
    tol = orth_tolerance(dtype, steps)
    for i in np.ndindex(ref.shape[:-2]):
        err = np.linalg.norm(got[i] - ref[i]) / np.linalg.norm(ref[i])
        assert err <= tol, (err, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (9, 1), (16, 16), (31, 33), (64, 64), (65, 63),
                                   (3, 40, 100), (2, 100, 40), (2, 2, 33, 64), (128, 128),
                                   (300, 129), (96, 1000), (517, 260)])
def test_orthogonalize(gpu, shape, dtype):
    rng = np.random.default_rng(sum(shape))
    G = stack(rng, shape, dtype)
    orth_close(g.orthogonalize(G), G, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(2100, 2100), (1100, 2500)])
def test_orthogonalize_large_tiles(gpu, shape, dtype):
    rng = np.random.default_rng(4)
    G = stack(rng, shape, dtype)
    orth_close(g.orthogonalize(G, steps=2), G, dtype, steps=2)


@pytest.mark.parametrize("steps", [0, 1, 3])
@pytest.mark.parametrize("dtype", DTYPES)
def test_orthogonalize_steps_and_polynomials(gpu, steps, dtype):
    rng = np.random.default_rng(6)
    for poly in (MUON, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0)):
        G = stack(rng, (70, 150), dtype)
        orth_close(g.orthogonalize(G, steps, poly), G, dtype, steps, poly)


def test_orthogonalize_makes_orthogonal(gpu):
    """The quintic with the fixed point at one, many steps: U V^T."""
    import torch
    rng = np.random.default_rng(8)
    G = stack(rng, (60, 90), "float32", 1.0)
    O = g.orthogonalize(G, steps=25, coefficients=(15 / 8, -10 / 8, 3 / 8))
    u, _, v = np.linalg.svd(host(G), full_matrices=False)
    assert np.abs(host(O) - u @ v).max() < 1e-4
    assert torch.allclose(O @ O.t(), torch.eye(60, device="cuda"), atol=1e-4)


@pytest.mark.parametrize("kind", ["dense", "transposed", "slice", "strided"])
@pytest.mark.parametrize("rows,cols", [(50, 90), (90, 50)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_orthogonalize_layouts_and_in_place(gpu, rows, cols, kind, dtype):
    import torch
    rng = np.random.default_rng(9)
    G = matrix(rng, rows, cols, dtype, kind)
    want = g.orthogonalize(G.contiguous())
    orth_close(want, G, dtype)
    for out_kind in ("dense", "transposed", "slice", "strided"):
        out = matrix(rng, rows, cols, dtype, out_kind)
        whole = out._base if out._base is not None else out
        before = whole.clone()
        assert g.orthogonalize(G, out=out) is out
        assert torch.equal(out, want)
        if out_kind in ("slice", "strided"):
            out.copy_(torch.as_strided(before, out.shape, out.stride(), out.storage_offset()))
            assert (whole == before).all()
    assert g.orthogonalize(G, out=G) is G
    assert torch.equal(G, want)


def test_orthogonalize_special_values(gpu):
    import torch
    for dtype in DTYPES:
        t = torch_type(dtype)
        G = torch.randn(4, 40, 50, device="cuda").to(t)
        G[1] = 0.0
        G[2, 7, 3] = math.inf
        G[3, 0, 0] = math.nan
        O = g.orthogonalize(G)
        assert (O[1] == 0).all()
        assert torch.isnan(O[2:]).all() and torch.isfinite(O[:2]).all()
        assert torch.equal(O[0], g.orthogonalize(G[0]))     # alone or in a stack
        assert torch.isnan(g.orthogonalize(G, steps=0)[2:]).all()
    for scale in (1e-35, 1e35):                             # the norm's square has no 32-bit value
        G = torch.randn(40, 50, device="cuda") * scale
        orth_close(g.orthogonalize(G, eps=0.0), G, "float32", eps=0.0)


def test_orthogonalize_repeats_bit_for_bit(gpu):
    import torch
    G = torch.randn(600, 400, device="cuda")
    first = g.orthogonalize(G)
    for _ in range(3):
        assert torch.equal(g.orthogonalize(G), first)


# ------------------------------------------------------- streams and graphs ---

def test_on_another_stream(gpu):
    import torch
    x, w = torch.randn(100, 300, device="cuda"), torch.randn(50, 300, device="cuda")
    want = g.mx_matmul(x, g.mx_quantize(w)), g.orthogonalize(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y, o = g.mx_matmul(x, g.mx_quantize(w)), g.orthogonalize(x)
    s.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(o, want[1])


def test_graph_replay_matches_eager(gpu):
    """Captured after an eager call on the same stream (which makes the
    workspace), replayed with new inputs and eager work in between."""
    import torch
    s = torch.cuda.Stream()
    x, w = torch.randn(100, 300, device="cuda"), torch.randn(50, 300, device="cuda")
    one = torch.randn(1, 300, device="cuda")

    def step():
        wq, wt = g.mx_quantize(w, "both")
        return (g.mx_matmul(x, wq), g.mx_matmul(one, wq), g.orthogonalize(w), wt.dequantize())

    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step()
        for i in range(4):
            for t in (x, w, one):
                t.copy_(torch.randn(t.shape, device="cuda"))
            want = [t.clone() for t in step()]
            s.synchronize()
            graph.replay()
            s.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b), i


def test_offsets_beyond_32_bits(gpu):
    """A packed matrix of more than 2^31 bytes of codes, and a C of more than
    2^32 elements apart."""
    import torch
    rows, cols = 1 << 20, 4160                # 2176 bytes a row
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, cols, device="cuda").to(x.dtype)
    q = g.mx_quantize(x)
    assert q.codes.numel() > 1 << 31
    tail = mx_values(host(x[-3:]))
    one = torch.randn(1, cols, device="cuda")
    y = g.mx_matmul(one, q)
    product_close(host(y[:, -3:]), mx_values(host(one)), tail, "float32")
    assert (y[:, :-3] == 0).all()
    del x
    big = torch.empty(40, 1 << 27, dtype=torch.bfloat16, device="cuda")
    C = big[:, :5]
    a = g.mx_quantize(torch.randn(40, 64, device="cuda"))
    b = g.mx_quantize(torch.randn(5, 64, device="cuda"))
    assert torch.equal(g.mx_matmul(a, b, C), g.mx_matmul(a, b, dtype=torch.bfloat16))


def test_linear_refuses_a_second_derivative(gpu):
    import torch
    x = torch.randn(9, 40, device=gpu, requires_grad=True)
    w = torch.randn(7, 40, device=gpu, requires_grad=True)
    y = g.mx_linear(x, w)
    first, = torch.autograd.grad(y, x, torch.ones_like(y), retain_graph=True)
    dx, = torch.autograd.grad(y, x, torch.ones_like(y, requires_grad=True), create_graph=True)
    assert torch.equal(first, dx)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(600, 600), (1100, 1210), (2310, 2200)])
def test_orthogonalize_many_tiles(gpu, shape, dtype):
    """Several bands of tile rows, the last one incomplete."""
    rng = np.random.default_rng(sum(shape))
    G = stack(rng, shape, dtype)
    orth_close(g.orthogonalize(G, steps=2), G, dtype, steps=2)


@pytest.mark.parametrize("shape", [(16, 16), (4000, 16), (64, 64), (130, 200), (256, 700)])
def test_orthogonalize_few_rows_in_two_parts(gpu, shape):
    """bf16 with a short side of 256 at most: two parts, so the result's own
    rounding (half a unit of each entry) is all that is left beside them."""
    rng = np.random.default_rng(sum(shape))
    G = stack(rng, shape, "bfloat16")
    got, ref = host(g.orthogonalize(G)), newton_schulz(host(G), 5, MUON, 1e-7)
    err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert err <= 12 * 5 * 2.0 ** -22 + HALF_ULP["bfloat16"]
