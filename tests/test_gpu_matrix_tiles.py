"""The matrix operators' tiles, slices and stacks (GPU): each test asks the
library which kernels its sizes take and says so where that changes.

Bounds are those of test_gpu_matrix.py; the references are formed in 64 bits
on the device (plain products) from values that mx_values and newton_schulz's
formulas give."""
import math
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_1607_00145_amd as g
from matrix_tiles import mx_tiles, orth_tiles
from test_gpu_matrix import HALF_ULP, MUON, orth_tolerance, torch_type

pytestmark = pytest.mark.gpu


def random_matrix(gen, rows, cols, dtype, kind="dense"):
    """Columns of many sizes, laid out as `kind` says."""
    import torch
    v = torch.randn(rows, cols, generator=gen, device="cuda")
    v *= torch.exp2(torch.randint(-4, 5, (1, cols), generator=gen, device="cuda").float())
    v = v.to(torch_type(dtype))
    if kind == "dense":
        return v
    if kind == "transposed":
        return v.t().contiguous().t()
    w = torch.full((rows, cols + 13), 7.0, dtype=v.dtype, device="cuda")   # slice
    w[:, 5:5 + cols] = v
    return w[:, 5:5 + cols]


def generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def values(q):
    """What a packed matrix stands for, in 64 bits (test_quantize_values has the
    packing itself)."""
    return q.dequantize().double()


def assert_product(got, a, b, dtype, alpha=1.0, beta=0.0, C=None):
    import torch
    bt = b.t().contiguous()
    ref, size = alpha * torch.mm(a, bt), abs(alpha) * torch.mm(a.abs(), bt.abs())
    if beta:
        ref, size = ref + beta * C, size + (beta * C).abs()
    bound = (a.shape[1] + 2) * 2.0 ** -24 * size + HALF_ULP[dtype] * 1.01 * ref.abs()
    if dtype == "float16":
        bound += 2.0 ** -24
    assert torch.isfinite(got).all()
    assert ((got.double() - ref).abs() <= bound).all()


# m, n, k: edge of the tiles, slices of the shared ones
PRODUCTS = {(3900, 3970, 2800): (256, 1), (4000, 3500, 777): (256, 1), (2000, 2500, 20000): (256, 3),
            (1500, 2600, 512): (128, 1), (2100, 4000, 8000): (128, 4), (777, 1250, 1999): (64, 1),
            (128, 128, 65537): (64, 13), (300, 700, 20000): (64, 4), (20, 3000, 4000): (0, 1)}


@pytest.mark.parametrize("kind", ["dense", "transposed", "slice"])
@pytest.mark.parametrize("size", list(PRODUCTS))
def test_product_tiles(gpu, size, kind):
    m, n, k = size
    swapped = kind == "transposed"            # C^T = B A^T: the same tiles the other way round
    t = mx_tiles(*((n, m, k) if swapped else size))
    if not swapped:
        assert (t.edge, t.slices) == PRODUCTS[size]
    elif size[0] > 32:
        assert t.edge == PRODUCTS[size][0]
    gen = generator(m + n + k)
    a, b = (g.mx_quantize(random_matrix(gen, r, k, "bfloat16")) for r in (m, n))
    for dtype, alpha, beta in (("float32", 1.0, 0.0), ("bfloat16", 0.75, -0.5)):
        C = random_matrix(gen, m, n, dtype, kind)
        before, whole = C.double(), C._base if kind == "slice" else None
        assert g.mx_matmul(a, b, C, alpha=alpha, beta=beta) is C
        assert_product(C, values(a), values(b), dtype, alpha, beta, before)
        if whole is not None:
            assert (whole[:, :5] == 7.0).all() and (whole[:, 5 + n:] == 7.0).all()


def linear_step(m, n, k, dtype="bfloat16"):
    import torch
    gen = generator(m + n + k)
    x, w = (random_matrix(gen, r, k, dtype).requires_grad_() for r in (m, n))
    dy = random_matrix(gen, m, n, dtype)
    y = g.mx_linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    pack = lambda t, along="cols": values(g.mx_quantize(t.detach(), along))
    assert_product(y.detach(), pack(x), pack(w), dtype)
    assert_product(dx, pack(dy), pack(w, "rows"), dtype)
    assert_product(dw, pack(dy, "rows"), pack(x, "rows"), dtype)


def test_gradients_of_one_launch_both_shared(gpu):
    """Two products in one launch, whose slots and counters follow one another."""
    m, n, k = 32700, 32600, 120
    t = mx_tiles(m, k, n), mx_tiles(n, k, m)
    assert [(x.edge, x.slices) for x in t] == [(128, 2), (128, 2)]
    linear_step(m, n, k)


@pytest.mark.parametrize("m,n,k,takes", [
    (16000, 130, 400, ((128, 1), (64, 7))), (16000, 300, 120, ((64, 1), (64, 7))),
    (3000, 2500, 2600, ((128, 1), (128, 1))), (16000, 20, 300, ((64, 1), (0, 1)))])
def test_gradients_in_tiles_of_their_own(gpu, m, n, k, takes):
    """dx and dw in two launches or in one where only dw is shared, and a dw of
    few rows."""
    assert tuple((t.edge, t.slices) for t in (mx_tiles(m, k, n), mx_tiles(n, k, m))) == takes
    linear_step(m, n, k)


def test_shared_sums_repeat_bit_for_bit(gpu):
    """Sums that several workgroups share do not depend on which comes last."""
    import torch
    gen = generator(5)
    for size in ((128, 128, 65537), (300, 700, 20000), (2100, 4000, 8000), (2000, 2500, 20000)):
        assert mx_tiles(*size).slices > 1
        a, b = (g.mx_quantize(random_matrix(gen, r, size[2], "bfloat16")) for r in size[:2])
        first = g.mx_matmul(a, b)
        for _ in range(4):
            assert torch.equal(g.mx_matmul(a, b), first)
    for shape in ((2100, 2100), (3000, 3500), (300, 16000)):
        assert max(t.slices for t in orth_tiles(1, *shape)) > 1
        G = random_matrix(gen, *shape, "float32")
        first = g.orthogonalize(G, steps=2)
        for _ in range(4):
            assert torch.equal(g.orthogonalize(G, steps=2), first)


# -------------------------------------------------------- orthogonalisation ---

def newton_schulz(G, steps, poly=MUON, eps=1e-7):
    """Of a stack [batch, rows, cols], in 64 bits."""
    import torch
    a, b, c = poly
    out = []
    for M in G.double():
        X = M if M.shape[0] <= M.shape[1] else M.t().contiguous()
        X = X / (X.square().sum().sqrt() + eps)
        for _ in range(steps):
            S = torch.mm(X, X.t().contiguous())
            X = a * X + torch.mm(b * S + c * torch.mm(S, S), X)
        out.append(X if M.shape[0] <= M.shape[1] else X.t())
    return torch.stack(out)


def assert_orthogonalized(got, ref, dtype, steps):
    import torch
    norm = torch.linalg.matrix_norm
    error = norm(got.double() - ref) / norm(ref)
    assert (error <= orth_tolerance(dtype if dtype != "bfloat16" else "float32", steps) +
            HALF_ULP[dtype]).all(), error


# rows, cols: edge and slices of S, b S + c S^2 and the update
SHAPES = {(4000, 4090): ((128, 8), (128, 9), (256, 1)), (3500, 3000): ((256, 3), (64, 4), (128, 3)),
          (2100, 2100): ((128, 3), (128, 3), (64, 7)), (2310, 2200): ((64, 4), (64, 4), (128, 1)),
          (300, 16000): ((64, 16), (32, 1), (128, 1)), (1000, 517): ((32, 1), (32, 1), (64, 1)),
          (600, 400): ((32, 1), (32, 1), (32, 1)), (96, 96): ((0, 1), (0, 1), (0, 1))}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_orthogonalize_tiles(gpu, shape, dtype):
    """Ragged edges, into rows, columns and a slice."""
    import torch
    assert tuple((t.edge, t.slices) for t in orth_tiles(1, *shape)) == SHAPES[shape]
    gen = generator(sum(shape))
    G = random_matrix(gen, *shape, dtype)
    ref = newton_schulz(G[None], 2)
    first = g.orthogonalize(G, steps=2)
    assert_orthogonalized(first[None], ref, dtype, 2)
    for kind in ("transposed", "slice"):
        out = random_matrix(gen, *shape, dtype, kind)
        assert torch.equal(g.orthogonalize(G, steps=2, out=out), first)
        if kind == "slice":
            assert (out._base[:, :5] == 7.0).all() and (out._base[:, 5 + shape[1]:] == 7.0).all()
    # S^2 is not formed where its coefficient is nothing
    cubic = (1.5, -0.5, 0.0)
    assert_orthogonalized(g.orthogonalize(G, 2, cubic)[None], newton_schulz(G[None], 2, cubic), dtype, 2)


STACKS = {(3, 300, 200): ((32, 1), (32, 1), (32, 1)), (20, 150, 200): ((32, 1), (32, 1), (64, 1)),
          (6, 700, 900): ((64, 1), (64, 1), (64, 1)), (4, 1100, 1000): ((64, 5), (64, 1), (128, 1)),
          (30, 400, 500): ((64, 1), (64, 1), (128, 1)), (3, 2500, 1500): ((128, 2), (128, 2), (128, 2)),
          (40, 96, 96): ((0, 1), (0, 1), (0, 1))}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", list(STACKS))
def test_orthogonalize_stacks_in_a_chain_of_launches(gpu, shape, dtype):
    """Stacks of matrices too large for one workgroup: contiguous, transposed, with
    gaps between them, and one of them NaN."""
    import torch
    assert tuple((t.edge, t.slices) for t in orth_tiles(*shape)) == STACKS[shape]
    gen = generator(sum(shape))
    b, r, c = shape
    G = random_matrix(gen, b * r, c, dtype).view(shape)
    ref = newton_schulz(G, 2)
    first = g.orthogonalize(G, steps=2)
    assert_orthogonalized(first, ref, dtype, 2)
    T = G.transpose(1, 2).contiguous().transpose(1, 2)
    # (the norm's squares are added in another order)
    assert_orthogonalized(g.orthogonalize(T, steps=2, out=torch.empty_like(T)), ref, dtype, 2)
    gaps = torch.full((b, r + 3, c), 7.0, dtype=G.dtype, device="cuda")
    gaps[:, :r] = G
    assert torch.equal(g.orthogonalize(gaps[:, :r], steps=2, out=gaps[:, :r]), first)
    assert (gaps[:, r:] == 7.0).all()
    G[1, r // 2, c // 3] = math.nan
    bad = g.orthogonalize(G, steps=2)
    assert torch.isnan(bad[1]).all()
    assert torch.equal(bad[0], first[0]) and torch.equal(bad[2:], first[2:])


# ------------------------------------------------------- threads and streams ---

def jobs(gen):
    """Calls that need the stream's workspace in different ways."""
    x = random_matrix(gen, 300, 20000, "bfloat16")
    w = g.mx_quantize(random_matrix(gen, 700, 20000, "bfloat16"))
    G, H = random_matrix(gen, 700, 900, "float32"), random_matrix(gen, 2100, 2100, "bfloat16")
    return [lambda: g.mx_matmul(x, w), lambda: g.orthogonalize(G, steps=2),
            lambda: g.orthogonalize(H, steps=1), lambda: g.mx_linear(x[:, :1000], x[:200, :1000])]


@pytest.mark.parametrize("shared", [False, True])
def test_calls_from_several_threads(gpu, shared):
    """Eight host threads, each on a stream of its own or all on one: the results
    of calls made one after the other."""
    import torch
    calls = jobs(generator(7))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    one = torch.cuda.Stream()
    # (streams of one thread's own: torch hands out 32 in turn)
    streams = [one if shared else torch.cuda.Stream() for _ in range(8)]

    def work(i):
        with torch.cuda.stream(streams[i]):
            got = [(j, calls[j]()) for j in [(i + s) % len(calls) for s in range(8)]]
        streams[i].synchronize()
        return got

    with ThreadPoolExecutor(8) as ex:
        for got in ex.map(work, range(8)):
            for j, t in got:
                assert torch.equal(t, want[j]), j
