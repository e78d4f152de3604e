"""Dropout, the linear layer and its gradients, routing, and the experts' products
against plain forms in 64 bits (layer_util.py) on one MI355X."""
import math

import numpy as np
import pytest
import torch

import layer_util as lu
import paper_1607_00145_amd as g

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def rand(seed, *shape, dtype=torch.float32, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=gen)).to(dtype)


# dropout ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 9), (2, 4096), (130, 1187),
                                       (257, 64), (1000, 1)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(gpu, dtype, rows, cols, p):
    x = rand(1, rows, cols, dtype=dtype).to(gpu)
    seed, offset = 0x123456789abcdef0 + rows, (7 << 32) + cols
    y = g.dropout(x, p, seed, offset)
    ref = x.double().cpu() * lu.mask(rows, cols, p, seed, offset)
    # one product in 32 bits with a factor that is itself rounded to 32
    lu.close(y, ref, 2 * lu.V * ref.abs() + lu.rounding(ref.abs() * (1 + 2 * lu.V), dtype))
    assert torch.equal(y == 0, (ref == 0).to(gpu))


def test_dropout_drops_what_it_says(gpu):
    x = torch.ones(4096, 4096, device=gpu)
    kept = float((g.dropout(x, 0.1, 5) != 0).float().mean())
    # 2^24 draws: five standard deviations
    assert abs(kept - (1 - 6554 / 65536)) < 5 * math.sqrt(0.09) / 4096


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_gradient_has_the_same_mask(gpu, dtype):
    x = rand(2, 33, 5, 77, dtype=dtype).to(gpu).requires_grad_()
    y = g.dropout(x, 0.3, 11, 3)
    dx, = torch.autograd.grad(y, x, torch.ones_like(y))
    assert torch.equal(dx != 0, y != 0)
    assert torch.equal(y, (x * dx.float()).to(dtype)) or dtype != torch.float32


def test_dropout_of_what_is_not_a_number(gpu):
    x = torch.full((64, 64), float("nan"), device=gpu)
    y = g.dropout(x, 0.5, 3)
    keep = lu.mask(64, 64, 0.5, 3, 0).to(gpu) != 0
    assert torch.equal(torch.isnan(y), keep) and bool((y[~keep] == 0).all())


def test_dropout_strides_and_in_place(gpu):
    base = rand(3, 50, 131).to(gpu)
    x = base[:, 3:100]
    y = g.dropout(x, 0.4, 9)
    assert torch.equal(y, g.dropout(x.contiguous(), 0.4, 9))
    assert torch.equal(g.dropout(base.t(), 0.4, 9), g.dropout(base.t().contiguous(), 0.4, 9))
    d = g.gett_dropout_t(0.4, 9, 0, None)
    st = g.gett_dropout(g.GETT_FLOAT32, 50, 97, x.data_ptr(), 131, d, x.data_ptr(), 131,
                        torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(x, y)
    assert torch.equal(base[:, :3], rand(3, 50, 131)[:, :3].to(gpu))


def test_no_dropout(gpu):
    """p = 0 is x itself; the C call copies."""
    x = rand(3, 50, 131).to(gpu).requires_grad_()
    assert g.dropout(x, 0.0, None) is x
    with pytest.raises(ValueError):
        g.dropout(x.detach().cpu(), 0.0, None)
    y, d = torch.empty_like(x), g.gett_dropout_t(0.0, 0, 0, None)
    st = g.gett_dropout(g.GETT_FLOAT32, 50, 131, x.data_ptr(), 131, d, y.data_ptr(), 131,
                        torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(x, y)


def test_dropout_seed_on_the_device(gpu):
    x = rand(4, 20, 40).to(gpu)
    seed = torch.tensor([-5], dtype=torch.int64, device=gpu)
    assert torch.equal(g.dropout(x, 0.5, seed, 2), g.dropout(x, 0.5, -5, 2))
    assert not torch.equal(g.dropout(x, 0.5, seed, 2), g.dropout(x, 0.5, seed, 3))


# linear ----------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 16, 64), (2, 7, 5), (33, 130, 72), (128, 128, 128), (129, 65, 200),
         (5, 1000, 515), (200, 96, 33), (64, 8, 1000), (300, 257, 136)]


def linear_case(seed, m, n, k, dtype, name):
    x, w = rand(seed, m, k, dtype=dtype), rand(seed + 1, n, k, dtype=dtype, scale=k ** -0.5)
    bias = rand(seed + 2, n, dtype=dtype, scale=0.3) if name != "relu" else None
    residual = rand(seed + 3, m, n, dtype=dtype) if name != "silu" else None
    return x, w, bias, residual


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", [None, "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear(gpu, dtype, name, m, n, k):
    x, w, bias, residual = linear_case(m + n, m, n, k, dtype, name)
    p = 0.25 if name == "gelu" else 0.0
    on = lambda t: None if t is None else t.to(gpu)
    y = g.linear(on(x), on(w), on(bias), activation=name, residual=on(residual), p=p, seed=42,
                 offset=6)
    ref, err, _, _ = lu.linear(x, w, bias, name, lu.mask(m, n, p, 42, 6), residual, dtype)
    lu.close(y, ref, err)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", [None, "gelu", "silu"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear_gradients(gpu, dtype, name, m, n, k):
    x, w, bias, residual = linear_case(m + n, m, n, k, dtype, name)
    dy = rand(m + 9, m, n, dtype=dtype)
    p = 0.25 if name != "silu" else 0.0
    leaves = [None if t is None else t.to(gpu).requires_grad_() for t in (x, w, bias, residual)]
    y = g.linear(leaves[0], leaves[1], leaves[2], activation=name, residual=leaves[3], p=p,
                 seed=42, offset=6)
    y.backward(dy.to(gpu))
    keep = lu.mask(m, n, p, 42, 6)
    ref, err, z, dz = lu.linear(x, w, bias, name, keep, residual, dtype)
    lu.close(y, ref, err, "y")
    grads = lu.linear_grads(dy, x, w, z, dz, name, keep, dtype)
    for what, leaf, (v, e) in zip(("dx", "dw", "dbias"), leaves, grads):
        if leaf is not None:
            lu.close(leaf.grad, v, e, what)
    if leaves[3] is not None:
        assert torch.equal(leaves[3].grad, dy.to(gpu))


def test_linear_relu_gradient(gpu):
    # (sums that are exact: where they are zero the slope is zero)
    x = torch.tensor([[1.0, -1.0], [2.0, 1.0], [-1.0, 0.0]], device=gpu, requires_grad=True)
    w = torch.tensor([[1.0, 1.0], [0.5, -1.0]], device=gpu, requires_grad=True)
    y = g.linear(x, w, activation="relu")
    ref = torch.relu(x.detach() @ w.detach().t())
    assert torch.equal(y.detach(), ref)
    dy = torch.tensor([[1.0, 2.0], [4.0, 8.0], [16.0, 32.0]], device=gpu)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    dz = dy * (ref > 0)
    assert torch.equal(dx, dz @ w.detach()) and torch.equal(dw, dz.t() @ x.detach())


# routing ---------------------------------------------------------------------

ROUTES = [(1, 4, 1, "softmax", False, 1, 1), (1, 64, 8, "softmax", False, 1, 1),
          (7, 64, 8, "sigmoid", True, 8, 3), (65, 200, 6, "sigmoid", True, 1, 1),
          (300, 256, 8, "softmax", True, 8, 4), (513, 33, 32, "softmax", False, 1, 1),
          (1000, 1024, 4, "sigmoid", True, 128, 40), (129, 512, 3, "softmax", False, 4, 1),
          (3000, 2, 2, "sigmoid", False, 1, 1)]


def check_route(r, ref, dtype_weights=True):
    weights, index, order, offsets, place = ref
    assert np.array_equal(r.index.cpu().numpy(), index)
    assert np.array_equal(r.order.cpu().numpy(), order)
    assert np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.place.cpu().numpy(), place)
    got = r.weights.detach().double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(weights))
    # scores in 64 bits, rounded once
    assert np.nanmax(np.abs(got - weights) - 2.0 ** -23 * np.abs(weights), initial=-1) <= 2.0 ** -149


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,e,k,scoring,biased,groups,kept", ROUTES)
@pytest.mark.parametrize("renormalize", [True, False])
def test_route(gpu, dtype, t, e, k, scoring, biased, groups, kept, renormalize):
    logits = rand(t + e, t, e, dtype=dtype)
    bias = rand(5, e, scale=0.1) if biased else None
    r = g.route(logits.to(gpu), k, scoring=scoring, bias=None if bias is None else bias.to(gpu),
                groups=groups, top_groups=kept, renormalize=renormalize, scale=1.5)
    check_route(r, lu.route(logits, k, scoring, bias, groups, kept, renormalize, 1.5))


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased,groups,kept", [(False, 1, 1), (True, 1, 1), (True, 4, 2)])
def test_route_ties_masks_and_nan(gpu, scoring, biased, groups, kept):
    inf = math.inf
    x = torch.zeros(9, 16)
    x[1] = torch.arange(16.0) % 3
    x[2, 3:] = -inf
    x[3] = -inf
    x[4, ::2] = -inf
    x[5, 7] = math.nan
    x[6] = math.nan
    x[7, 5] = inf
    x[8, 1:] = torch.finfo(torch.float32).min
    bias = (torch.arange(16) % 2).float() * 0.25 if biased else None
    r = g.route(x.to(gpu), 4, scoring=scoring, bias=None if bias is None else bias.to(gpu),
                groups=groups, top_groups=kept)
    check_route(r, lu.route(x, 4, scoring, bias, groups, kept))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,e,k,scoring,biased,groups,kept", ROUTES)
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_gradient(gpu, dtype, t, e, k, scoring, biased, groups, kept, renormalize):
    logits, dw = rand(t + e, t, e, dtype=dtype), rand(3, t, k)
    bias = rand(5, e, scale=0.1) if biased else None
    x = logits.to(gpu).requires_grad_()
    r = g.route(x, k, scoring=scoring, bias=None if bias is None else bias.to(gpu), groups=groups,
                top_groups=kept, renormalize=renormalize, scale=1.5)
    dx, = torch.autograd.grad(r.weights, x, dw.to(gpu))
    v = logits.double().requires_grad_()
    s = torch.softmax(v, 1) if scoring == "softmax" else torch.sigmoid(v)
    c = s.gather(1, r.index.cpu().long())
    w = 1.5 * (c / c.sum(1, keepdim=True) if renormalize else c)
    ref, = torch.autograd.grad(w, v, dw.double())
    # 64 bits to 32 (once or twice), to the type; cancellation of terms of dw's size
    # is at 2^-53 and below
    err = 4 * lu.V * ref.abs() + 1e-14 * dw.double().abs().sum(1, keepdim=True)
    lu.close(dx, ref, err + lu.rounding(ref.abs() + err, dtype))


@pytest.mark.parametrize("e,groups", [(8, 1), (8, 2), (9, 3), (1024, 1)])
def test_route_far_below_the_largest(gpu, e, groups):
    """The bias or the groups take experts whose scores vanish beside the token's largest:
    renormalised weights and their gradient are still those of the chosen."""
    logits = rand(3, 5, e)
    logits[:, 0] += 2000.0
    bias = torch.zeros(e)
    bias[0], bias[e - 2:] = -10.0, 5.0
    x = logits.to(gpu).requires_grad_()
    r = g.route(x, 2, bias=bias.to(gpu), groups=groups, top_groups=1)
    check_route(r, lu.route(logits, 2, "softmax", bias, groups, 1))
    assert float((r.weights.detach().sum(1) - 1).abs().max()) <= 2 * lu.V
    dw = rand(4, 5, 2)
    dx, = torch.autograd.grad(r.weights, x, dw.to(gpu))
    v = logits.double().requires_grad_()
    w = torch.softmax(v.gather(1, r.index.cpu().long()), 1)
    ref, = torch.autograd.grad(w, v, dw.double())
    err = 4 * lu.V * ref.abs() + 1e-14 * dw.double().abs().sum(1, keepdim=True)
    lu.close(dx, ref, err + lu.rounding(ref.abs() + err, torch.float32))


def test_route_of_no_tokens(gpu):
    r = g.route(torch.empty(0, 8, device=gpu), 2)
    assert r.weights.shape == (0, 2) and r.order.numel() == 0
    assert r.offsets.tolist() == [0] * 9


# experts ---------------------------------------------------------------------

EXPERTS = [(1, 4, 2, 16, 8), (5, 8, 3, 33, 17), (64, 4, 2, 64, 128), (130, 6, 2, 96, 40),
           (300, 3, 1, 128, 72), (40, 64, 8, 72, 136)]


def experts_case(seed, t, e, k, width, n, dtype):
    logits = rand(seed, t, e) + rand(seed + 1, 1, e)
    return (logits, rand(seed + 2, t, width, dtype=dtype),
            rand(seed + 3, e, n, width, dtype=dtype, scale=width ** -0.5),
            rand(seed + 4, e, n, dtype=dtype, scale=0.3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,e,k,width,n", EXPERTS)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("name", [None, "gelu", "silu"])
def test_expert_linear(gpu, dtype, t, e, k, width, n, gather, name):
    logits, x, w, bias = experts_case(t, t, e, k, width, n, dtype)
    logits[t // 2] = -math.inf              # a token without experts
    r = g.route(logits.to(gpu), k)
    order, offsets = r.order.cpu().long(), r.offsets.cpu().tolist()
    if not gather:
        x = rand(7, t * k, width, dtype=dtype)
    dy = rand(8, t * k, n, dtype=dtype)
    leaves = [v.to(gpu).requires_grad_() for v in (x, w, bias)]
    y = g.expert_linear(leaves[0], leaves[1], r, leaves[2], activation=name, gather=gather)
    dx, dw, db = torch.autograd.grad(y, leaves, dy.to(gpu))
    live = offsets[-1]
    assert not y[live:].any()
    ref_dx, err_dx = torch.zeros(x.shape, dtype=torch.float64), torch.zeros(x.shape, dtype=torch.float64)
    for i in range(e):
        a, b = offsets[i], offsets[i + 1]
        rows = order[a:b] // k if gather else torch.arange(a, b)
        keep = torch.ones(b - a, n, dtype=torch.float64)
        ref, err, z, dz = lu.linear(x[rows], w[i], bias[i], name, keep, None, dtype)
        lu.close(y[a:b], ref, err, f"y {i}")
        grads = lu.linear_grads(dy[a:b], x[rows], w[i], z, dz, name, keep, dtype)
        lu.close(dw[i], *grads[1], f"dw {i}")
        lu.close(db[i], *grads[2], f"db {i}")
        ref_dx.index_add_(0, rows, grads[0][0])
        err_dx.index_add_(0, rows, grads[0][1] + k * lu.V * grads[0][0].abs())
    lu.close(dx, ref_dx, err_dx + lu.rounding(ref_dx.abs() + err_dx, dtype), "dx")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("t,e,k,cols", [(1, 2, 1, 1), (9, 8, 8, 100), (70, 5, 2, 515), (33, 40, 6, 1024)])
def test_combine(gpu, dtype, wide, t, e, k, cols):
    logits = rand(1, t, e)
    logits[t // 2] = -math.inf
    r = g.route(logits.to(gpu), k)
    place = r.place.cpu().long()
    h, dy = rand(2, t * k, cols, dtype=dtype), rand(3, t, cols, dtype=dtype)
    wtype = torch.float32 if wide else dtype
    weights, residual = rand(4, t, k, dtype=wtype), rand(5, t, cols, dtype=dtype)
    leaves = [v.to(gpu).requires_grad_() for v in (h, weights, residual)]
    y = g.combine(leaves[0], r, weights=leaves[1], residual=leaves[2])
    dh, dw, dres = torch.autograd.grad(y, leaves, dy.to(gpu))
    there = (place >= 0).double()
    mine = h.double()[place.clamp(min=0)] * there[..., None]
    terms = weights.double()[..., None] * mine
    ref, size = residual.double() + terms.sum(1), residual.double().abs() + terms.abs().sum(1)
    err = (k + 2) * lu.V * size
    lu.close(y, ref, err + lu.rounding(ref.abs() + err, dtype), "y")
    assert torch.equal(dres, dy.to(gpu))
    prods = dy.double()[:, None] * mine
    err = (cols + 2) * lu.V * prods.abs().sum(2)
    lu.close(dw, prods.sum(2), err + lu.rounding(prods.sum(2).abs() + err, wtype), "dw")
    ref = torch.zeros(h.shape, dtype=torch.float64)
    for i, j in (place >= 0).nonzero().tolist():
        ref[place[i, j]] = weights[i, j].double() * dy[i].double()
    lu.close(dh, ref, 2 * lu.V * ref.abs() + lu.rounding(ref.abs() * (1 + 2 * lu.V), dtype), "dh")


def test_run_of_the_operators_together(gpu):
    """A layer of experts with dropout and a residual, forward and backward, against
    the same in torch on 64-bit copies."""
    t, e, k, d, h = 96, 6, 2, 64, 80
    x, router = rand(1, t, d), rand(2, e, d, scale=d ** -0.5)
    w1, w2 = rand(3, e, h, d, scale=d ** -0.5), rand(4, e, d, h, scale=h ** -0.5)
    wo, dy = rand(5, d, d, scale=d ** -0.5), rand(6, t, d)
    leaves = [v.to(gpu).requires_grad_() for v in (x, router, w1, w2, wo)]
    lx, lr, l1, l2, lo = leaves
    r = g.route(g.linear(lx, lr), k)
    a = g.expert_linear(lx, l1, r, activation="silu", gather=True)
    m = g.combine(g.expert_linear(a, l2, r), r, residual=lx)
    y = g.linear(g.dropout(m, 0.2, 5), lo, activation="gelu", residual=lx, p=0.1, seed=6)
    got = torch.autograd.grad(y, leaves, dy.to(gpu))
    vx, vr, v1, v2, vo = (v.double().requires_grad_() for v in (x, router, w1, w2, wo))
    p = torch.softmax(vx @ vr.t(), 1)
    index = r.index.cpu().long()
    assert torch.equal(index, p.topk(k, 1)[1])
    c = p.gather(1, index)
    c = c / c.sum(1, keepdim=True)
    out = vx
    for j in range(k):
        a = torch.nn.functional.silu(torch.einsum("td,thd->th", vx, v1[index[:, j]]))
        out = out + c[:, j:j + 1] * torch.einsum("th,tdh->td", a, v2[index[:, j]])
    out = out * lu.mask(t, d, 0.2, 5, 0)
    ref = vx + torch.nn.functional.gelu(out @ vo.t()) * lu.mask(t, d, 0.1, 6, 0)
    want = torch.autograd.grad(ref, (vx, vr, v1, v2, vo), dy.double())
    # six products deep, each within (K + 4) 2^-24 of sums of some sqrt(K) times its
    # size: 6 * 100 * 10 * 2^-24
    tol = 6000 * 2.0 ** -24
    for a, b in zip((y, *got), (ref, *want)):
        off = (a.detach().double().cpu() - b.detach()).norm() / b.detach().norm()
        assert float(off) < tol
