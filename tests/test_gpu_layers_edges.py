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


def wider(t, more):
    """A matrix of t's shape in rows that are `more` numbers wider, those of 7."""
    base = torch.full((t.shape[0], t.shape[1] + more), 7.0, dtype=t.dtype, device=t.device)
    view = base[:, :t.shape[1]]
    view.copy_(t)
    return base, view


def drop_of(p, seed):
    return g.gett_dropout_t(p, seed, 0, None)


@pytest.mark.parametrize("more", [0, 5])
@pytest.mark.parametrize("dtype,m,n,k,edge,shared", [
    (torch.bfloat16, 8300, 7900, 328, 256, False), (torch.bfloat16, 4487, 4507, 4104, 256, True),
    (torch.float16, 3085, 2579, 40, 128, False), (torch.bfloat16, 2317, 3380, 4104, 128, True),
    (torch.float16, 3789, 1070, 520, 64, False), (torch.bfloat16, 4151, 97, 4104, 64, True),
    (torch.bfloat16, 4165, 197, 328, 32, False), (torch.float32, 2525, 3276, 40, 128, False),
    (torch.float32, 353, 3403, 4104, 128, True), (torch.float32, 3691, 611, 1032, 64, True),
    (torch.float32, 201, 145, 40, 32, False), (torch.float16, 1, 700, 264, 0, False),
    (torch.float32, 3, 700, 261, 0, False)])
def test_residual_in_place(gpu, dtype, m, n, k, edge, shared, more):
    """Y may be the residual itself: the same result, bit by bit, in every kind of tile."""
    t = product_tiles(CODES[dtype], m, n, k)
    assert t.edge == edge and (t.slices > 1) == shared
    x, w, bias = (on_gpu(v) for v in (rand(1, m, k, dtype=dtype), rand(2, n, k, dtype=dtype, scale=k ** -0.5),
                                      rand(3, n, dtype=dtype)))
    residual = rand(4, m, n, dtype=dtype).to(gpu)
    want = g.linear(x, w, bias, activation="gelu", residual=residual, p=0.25, seed=9)
    base, y = wider(residual, more)
    st = g.gett_linear(CODES[dtype], m, n, k, x.data_ptr(), k, w.data_ptr(), k, bias.data_ptr(), 2,
                       drop_of(0.25, 9), y.data_ptr(), n + more, 0, n, y.data_ptr(), n + more,
                       torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert torch.equal(y, want) and bool((base[:, n:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [5, 32])
def test_residual_in_place_of_few_rows(gpu, dtype, m):
    """The same of rows that a weight at an odd address is multiplied with."""
    n, k = 70, 203
    x, bias = rand(1, m, k, dtype=dtype).to(gpu), rand(3, n, dtype=dtype).to(gpu)
    w = rand(2, n, k + 2, dtype=dtype).to(gpu)[:, 1:k + 1]
    residual = rand(4, m, n, dtype=dtype).to(gpu)
    want = g.linear(x, w, bias, activation="silu", residual=residual)
    y = residual.clone()
    st = g.gett_linear(CODES[dtype], m, n, k, x.data_ptr(), k, w.data_ptr(), k + 2, bias.data_ptr(), 3, None,
                       y.data_ptr(), n, 0, n, y.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,e,k,cols,more", [(1, 2, 1, 1, 0), (9, 8, 8, 100, 3), (70, 5, 2, 515, 0),
                                             (333, 40, 6, 1024, 8)])
def test_combine_in_place(gpu, dtype, t, e, k, cols, more):
    logits = rand(1, t, e)
    logits[t // 2] = -math.inf
    r = g.route(logits.to(gpu), k)
    h, residual = rand(2, t * k, cols, dtype=dtype).to(gpu), rand(5, t, cols, dtype=dtype).to(gpu)
    want = g.combine(h, r, residual=residual)
    base, y = wider(residual, more)
    st = g.gett_combine(CODES[dtype], t, k, cols, h.data_ptr(), cols, g.GETT_FLOAT32, r.weights.data_ptr(),
                        r.place.data_ptr(), y.data_ptr(), cols + more, y.data_ptr(), cols + more,
                        torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert torch.equal(y, want) and bool((base[:, cols:] == 7).all())


# dropout ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("p", [0.1, 0.3, 0.5])
def test_dropout_and_its_gradient_number_by_number(gpu, dtype, p):
    """One product in 32 bits with the mask's factor in 32 bits, rounded once."""
    rows, cols = 165, 77
    factor = lu.mask(rows, cols, p, 11, 3).float().to(gpu)
    x, dy = rand(2, rows, cols, dtype=dtype).to(gpu).requires_grad_(), rand(3, rows, cols, dtype=dtype).to(gpu)
    y = g.dropout(x, p, 11, 3)
    dx, = torch.autograd.grad(y, x, dy)
    assert torch.equal(y.detach(), (x.detach().float() * factor).to(dtype))
    assert torch.equal(dx, (dy.float() * factor).to(dtype))


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


# memory ----------------------------------------------------------------------

@pytest.mark.parametrize("apart", [(1 << 23) - 8, 1 << 23, (1 << 23) + 8])
def test_rows_far_apart(gpu, apart):
    """Rows of 16 bits 16 MB apart, about as far as a tile reaches them where they lie."""
    m, n, k = 260, 40, 72
    x, w, dy = (rand(i, *s, dtype=torch.bfloat16).to(gpu) for i, s in ((1, (m, k)), (2, (n, k)), (3, (m, n))))
    far = torch.empty(m * apart, dtype=torch.bfloat16, device=gpu).as_strided((m, k), (apart, 1))
    far.copy_(x)
    results = []
    for v in (x, far):
        leaves = [v.detach().requires_grad_(), w.detach().requires_grad_()]
        y = g.linear(*leaves)
        results.append([y.detach(), *torch.autograd.grad(y, leaves, dy)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    for v in (dy, torch.empty(m * apart, dtype=torch.bfloat16, device=gpu).as_strided((m, n), (apart, 1)).copy_(dy)):
        leaves = [x.detach().requires_grad_(), w.detach().requires_grad_()]
        results.append(list(torch.autograd.grad(g.linear(*leaves), leaves, v)))
    assert all(torch.equal(a, b) for a, b in zip(results[2], results[3]))


@pytest.mark.parametrize("t", [(1 << 20) + 3, (1 << 21) - 9])
def test_gathered_rows_beyond_4_gb(gpu, t):
    """Tokens of more than 2^32 bytes: the last ones' rows are theirs."""
    d, n, e = 2048, 24, 3
    x = torch.empty(t, d, dtype=torch.bfloat16, device=gpu)
    x[:] = torch.arange(t, device=gpu)[:, None] % 127      # (whole numbers: 16 bits hold them)
    w = torch.zeros(e, n, d, dtype=torch.bfloat16, device=gpu)
    w[:, :, 0] = torch.arange(1, e + 1, device=gpu)[:, None]
    logits = torch.zeros(t, e, device=gpu)
    logits[torch.arange(t, device=gpu), torch.arange(t, device=gpu) % e] = 5.0
    r = g.route(logits, 1)
    y = g.expert_linear(x, w, r, gather=True)
    back = g.combine(y, r, weights=torch.ones(t, 1, device=gpu))
    token = torch.arange(t, device=gpu)
    want = (token % 127).float() * (token % e + 1)
    # (up to 378: bf16 holds every second one of those beyond 256)
    assert torch.equal(back.float(), want.to(torch.bfloat16).float()[:, None].expand(t, n))


# one gradient without the others -------------------------------------------------

def subsets(n):
    return [[i for i in range(n) if bits >> i & 1] for bits in range(1, 1 << n)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name,p", [(None, 0.0), (None, 0.3), ("gelu", 0.3)])
@pytest.mark.parametrize("m,n,k", [(1, 24, 40), (37, 51, 29), (300, 136, 264)])
def test_every_choice_of_gradients(gpu, dtype, name, p, m, n, k):
    tensors = [v.to(gpu) for v in (rand(1, m, k, dtype=dtype), rand(2, n, k, dtype=dtype, scale=k ** -0.5),
                                   rand(3, n, dtype=dtype), rand(5, m, n, dtype=dtype))]
    dy = rand(4, m, n, dtype=dtype).to(gpu)

    def gradients(wanted):
        leaves = [t.detach().requires_grad_(i in wanted) for i, t in enumerate(tensors)]
        y = g.linear(*leaves[:3], activation=name, residual=leaves[3], p=p, seed=3)
        return torch.autograd.grad(y, [leaves[i] for i in wanted], dy)

    every = gradients(range(4))
    for wanted in subsets(4):
        assert all(torch.equal(v, every[i]) for i, v in zip(wanted, gradients(wanted))), wanted


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("t,e,k,width,n", [(1, 4, 2, 40, 24), (90, 6, 2, 77, 51), (700, 4, 2, 520, 264),
                                           (2000, 8, 1, 256, 512)])
def test_every_choice_of_the_experts_gradients(gpu, dtype, gather, t, e, k, width, n):
    logits = rand(1, t, e)
    logits[t // 2] = -math.inf
    r = g.route(logits.to(gpu), k)
    tensors = [v.to(gpu) for v in (rand(2, t if gather else t * k, width, dtype=dtype),
                                   rand(3, e, n, width, dtype=dtype, scale=width ** -0.5), rand(4, e, n, dtype=dtype))]
    dy = rand(5, t * k, n, dtype=dtype).to(gpu)

    def gradients(wanted):
        leaves = [v.detach().requires_grad_(i in wanted) for i, v in enumerate(tensors)]
        y = g.expert_linear(leaves[0], leaves[1], r, leaves[2], activation="silu", gather=gather)
        return torch.autograd.grad(y, [leaves[i] for i in wanted], dy)

    every = gradients(range(3))
    for wanted in subsets(3):
        assert all(torch.equal(v, every[i]) for i, v in zip(wanted, gradients(wanted))), wanted
    h, weights, residual = (rand(i, *s, dtype=dtype).to(gpu) for i, s in ((6, (t * k, n)), (7, (t, k)), (8, (t, n))))
    back = rand(9, t, n, dtype=dtype).to(gpu)

    def combined(wanted):
        leaves = [v.detach().requires_grad_(i in wanted) for i, v in enumerate((h, weights, residual))]
        y = g.combine(leaves[0], r, weights=leaves[1], residual=leaves[2])
        return torch.autograd.grad(y, [leaves[i] for i in wanted], back)

    every = combined(range(3))
    for wanted in subsets(3):
        assert all(torch.equal(v, every[i]) for i, v in zip(wanted, combined(wanted))), wanted


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("t,width,n", [(1, 0, 8), (50, 0, 24), (50, 16, 0), (300, 0, 40), (0, 8, 16)])
def test_experts_of_empty_extents(gpu, dtype, gather, t, width, n):
    e, k = 3, 2
    r = g.route(rand(1, t, e).to(gpu), k)
    x = torch.zeros(t if gather else t * k, width, dtype=dtype, device=gpu).requires_grad_()
    w = torch.zeros(e, n, width, dtype=dtype, device=gpu).requires_grad_()
    b = rand(2, e, n, dtype=dtype).to(gpu).requires_grad_()
    y = g.expert_linear(x, w, r, b, activation="relu", gather=gather)
    expert = torch.repeat_interleave(torch.arange(e, device=gpu), r.offsets.diff().long())
    assert torch.equal(y, b.detach().relu()[expert])
    dx, dw, db = torch.autograd.grad(y, (x, w, b), torch.ones_like(y))
    assert dx.shape == x.shape and dw.shape == w.shape and not dx.any() and not dw.any()
    count = r.offsets.diff()[:, None].to(dtype)
    assert torch.equal(db, torch.where(b.detach() > 0, count, torch.zeros_like(count)))
    assert torch.equal(g.combine(y, r, weights=torch.ones(t, k, device=gpu)).float(),
                       torch.zeros(t, n, device=gpu) if not t or not n else
                       (y.detach().float()[r.place.long()].sum(1).to(dtype).float()))


# numbers that are none, in places that do not count -----------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("t,e,k,width,n", [(9, 4, 2, 40, 24), (40, 16, 2, 77, 51), (130, 6, 2, 64, 72),
                                           (700, 4, 2, 520, 264)])
def test_nan_of_tokens_without_experts(gpu, dtype, gather, t, e, k, width, n):
    """Rows of no expert, and gradients of such, are not read into anybody's sums."""
    logits = rand(1, t, e)
    logits[1::3] = -math.inf
    r = g.route(logits.to(gpu), k)
    live = int(r.offsets[-1])
    w, b = rand(3, e, n, width, dtype=dtype).to(gpu), rand(4, e, n, dtype=dtype).to(gpu)
    x, dy = rand(2, t if gather else t * k, width, dtype=dtype).to(gpu), rand(5, t * k, n, dtype=dtype).to(gpu)
    back = rand(6, t, n, dtype=dtype).to(gpu)
    results = []
    for bad in (0.0, math.nan, math.inf):
        x, dy, back = x.clone(), dy.clone(), back.clone()
        if gather:
            x[1::3] = bad
        else:
            x[live:] = bad
        dy[live:] = bad
        leaves = [v.detach().requires_grad_() for v in (x, w, b)]
        y = g.expert_linear(leaves[0], leaves[1], r, leaves[2], activation="gelu", gather=gather)
        out = [y.detach(), *torch.autograd.grad(y, leaves, dy)]
        h = y.detach().clone()
        h[live:] = bad
        back[1::3] = bad
        more = [h.requires_grad_(), r.weights.detach().requires_grad_()]
        z = g.combine(more[0], r, weights=more[1])
        dh, dw = torch.autograd.grad(z, more, back)
        results.append(out + [z.detach(), dh, dw])
    for other in results[1:]:
        for i, (a, c) in enumerate(zip(results[0], other)):
            assert not c.isnan().any() and torch.equal(a, c), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 70, 40), (20, 70, 41), (150, 96, 72), (300, 260, 264)])
def test_nan_of_one_row_stays_in_it(gpu, dtype, m, n, k):
    x, w, b = rand(1, m, k, dtype=dtype).to(gpu), rand(2, n, k, dtype=dtype).to(gpu), rand(3, n, dtype=dtype).to(gpu)
    dy, row = rand(4, m, n, dtype=dtype).to(gpu), m // 2
    want = g.linear(x, w, b, activation="silu")
    x[row, k - 1] = math.nan
    leaf = x.requires_grad_()
    y = g.linear(leaf, w, b, activation="silu")
    dx, = torch.autograd.grad(y, leaf, dy)
    others = torch.arange(m, device=gpu) != row
    assert y[row].isnan().all() and torch.equal(y[others], want[others])
    assert dx[row].isnan().all() and not dx[others].isnan().any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 70, 40), (20, 70, 41), (300, 260, 264)])
def test_gradients_that_are_dropped_do_not_count(gpu, dtype, m, n, k):
    x, w, b = rand(1, m, k, dtype=dtype).to(gpu), rand(2, n, k, dtype=dtype).to(gpu), rand(3, n, dtype=dtype).to(gpu)
    dy = rand(4, m, n, dtype=dtype).to(gpu)
    keep = lu.mask(m, n, 0.5, 7, 0).to(gpu) != 0
    results = []
    for bad in (0.0, math.nan, math.inf):
        leaves = [v.detach().requires_grad_() for v in (x, w, b)]
        y = g.linear(*leaves, activation="gelu", p=0.5, seed=7)
        results.append(torch.autograd.grad(y, leaves, torch.where(keep, dy, torch.full_like(dy, bad))))
    for other in results[1:]:
        assert all(torch.equal(a, c) for a, c in zip(results[0], other))
