"""The layers' operators where they can go wrong beside their arithmetic: every kind of
tile, shared sums, odd strides and addresses, uneven experts, repeated calls, streams,
graphs, large offsets, refusals."""
import math
import threading

import pytest
import torch

import layer_util as lu
import paper_1607_00145_amd as g
from test_gpu_layers import rand
from test_layers_abi import product_tiles

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODES = {torch.float32: g.GETT_FLOAT32, torch.bfloat16: g.GETT_BFLOAT16, torch.float16: g.GETT_FLOAT16}

# m, n, k and what they have to take: the tiles' edge, whether sums are shared, and
# whether workgroups are alone on a CU (-1), all resident at once (0) or more (1)
TILES16 = [(4372, 2693, 72, 256, False, -1), (8300, 7900, 328, 256, False, 1), (4487, 4507, 4104, 256, True, 1),
           (1122, 1805, 40, 128, False, -1), (3237, 1229, 40, 128, False, 0), (3085, 2579, 40, 128, False, 1),
           (2317, 3380, 4104, 128, True, 1),
           (4897, 130, 1032, 64, False, -1), (260, 3645, 40, 64, False, 0), (3789, 1070, 520, 64, False, 1),
           (4151, 97, 4104, 64, True, 0),
           (86, 228, 40, 32, False, -1), (4213, 40, 40, 32, False, 0), (4165, 197, 328, 32, False, 1)]
TILES32 = [(2502, 1219, 40, 128, False, -1), (2596, 1571, 40, 128, False, 0), (2525, 3276, 40, 128, False, 1),
           (353, 3403, 4104, 128, True, -1), (609, 2450, 4104, 128, True, 0), (3820, 4384, 520, 128, True, 1),
           (4914, 291, 40, 64, False, 0), (4708, 790, 40, 64, False, 1),
           (40, 41, 4104, 64, True, -1), (4355, 39, 2056, 64, True, 0), (3691, 611, 1032, 64, True, 1),
           (129, 4964, 40, 64, False, -1), (201, 145, 40, 32, False, -1), (4213, 40, 40, 32, False, 0), (2696, 707, 40, 32, False, 1)]


def on_gpu(t):
    return None if t is None else t.to("cuda")


def linear64(x, w, bias, name, residual, dtype):
    """y and its error's bound as layer_util.linear has them, on the device."""
    x, w = x.cuda().double(), w.cuda().double()
    z, size = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
    if bias is not None:
        z, size = z + bias.cuda().double(), size + bias.cuda().double().abs()
    a = lu.act(name, z)[0]
    r = 0.0 if residual is None else residual.cuda().double()
    err = 1.14 * (x.shape[1] + 4) * lu.V * size + (lu.act_error(z) * z.abs() if name else 0)
    y = a + r
    err = err + 4 * lu.V * (a.abs() + (r.abs() if residual is not None else 0))
    return y, err + lu.rounding(y.abs() + err, dtype)


def close(got, ref, err, what=""):
    bad = ~((got.double() - ref).abs() <= err)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("dtype,m,n,k,edge,shared,fill", [(torch.bfloat16, *t) for t in TILES16] +
                         [(torch.float16, *TILES16[0])] + [(torch.float32, *t) for t in TILES32])
def test_every_kind_of_tile(gpu, dtype, m, n, k, edge, shared, fill):
    t = product_tiles(CODES[dtype], m, n, k)
    resident = {256: 256, 32: 768}.get(edge, 512)
    assert t.edge == edge and (t.slices > 1) == shared
    assert fill == (-1 if t.workgroups <= 256 else 0 if t.workgroups <= resident else 1)
    x, w = rand(1, m, k, dtype=dtype), rand(2, n, k, dtype=dtype, scale=k ** -0.5)
    bias, residual = rand(3, n, dtype=dtype), rand(4, m, n, dtype=dtype)
    leaves = [on_gpu(v).requires_grad_() for v in (x, w, bias, residual)]
    y = g.linear(leaves[0], leaves[1], leaves[2], activation="silu", residual=leaves[3])
    close(y.detach(), *linear64(x, w, bias, "silu", residual, dtype), "y")
    # the gradients' tiles: each product against 64 bits, dz being exact (no activation)
    dy = rand(5, m, n, dtype=dtype).cuda()
    plain = g.linear(leaves[0], leaves[1])
    dx, dw = torch.autograd.grad(plain, leaves[:2], dy)
    for got, a, b in ((dx, dy, w.cuda()), (dw, dy.t(), x.cuda())):
        a, b = a.double().contiguous(), b.double()
        ref = a @ b
        err = (a.shape[1] + 2) * lu.V * (a.abs() @ b.abs())
        close(got, ref, err + lu.rounding(ref.abs() + err, dtype), "gradient")
    again = torch.autograd.grad(g.linear(leaves[0], leaves[1]), leaves[:2], dy)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 32, 33, 64, 65])
@pytest.mark.parametrize("n,k", [(31, 7), (70, 1030), (33, 4104), (8200, 72)])
def test_few_rows(gpu, dtype, m, n, k):
    x, w = rand(m, m, k, dtype=dtype), rand(2, n, k, dtype=dtype, scale=k ** -0.5)
    bias, residual = rand(3, n, dtype=dtype), rand(4, m, n, dtype=dtype)
    y = g.linear(on_gpu(x), on_gpu(w), on_gpu(bias), activation="gelu", residual=on_gpu(residual))
    close(y, *linear64(x, w, bias, "gelu", residual, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [3, 20, 150])
def test_strides_and_addresses(gpu, dtype, m):
    """Slices of wide matrices at odd addresses, transposed and broadcast operands."""
    wide_x, wide_w = rand(1, m, 215, dtype=dtype).cuda(), rand(2, 90, 300, dtype=dtype).cuda()
    x, w, res = wide_x[:, 3:203], wide_w[:, 7:207], rand(3, 90, m, dtype=dtype).cuda().t()
    bias = rand(4, 1, dtype=dtype).cuda().expand(90)
    # (few rows of weights at odd addresses are summed in another order than on the grid)
    want = linear64(x, w, bias, None, res, dtype)
    close(g.linear(x.contiguous(), w.contiguous(), bias.contiguous(), residual=res.contiguous()), *want)
    close(g.linear(x, w, bias, residual=res), *want)
    assert torch.equal(g.linear(x, w, bias, residual=res), g.linear(x, w, bias, residual=res))
    leaves = [v.detach().requires_grad_() for v in (wide_x, wide_w)]
    dy = rand(5, 90, m, dtype=dtype).cuda().t()
    grads = torch.autograd.grad(g.linear(leaves[0][:, 3:203], leaves[1][:, 7:207]), leaves, dy)
    flat = [v.contiguous().requires_grad_() for v in (x.detach(), w.detach())]
    ref = torch.autograd.grad(g.linear(*flat), flat, dy.contiguous())
    assert torch.equal(grads[0][:, 3:203], ref[0]) and torch.equal(grads[1][:, 7:207], ref[1])
    assert not grads[0][:, :3].any() and not grads[1][:, 207:].any()
    # one row for all: its gradient is the sum
    one = rand(6, 1, 200, dtype=dtype).cuda().requires_grad_()
    d1, = torch.autograd.grad(g.linear(one.expand(m, 200), w), one, dy)
    full = torch.autograd.grad(g.linear((t := one.detach().repeat(m, 1).requires_grad_()), w), t, dy)[0]
    assert torch.equal(d1, full.sum(0, keepdim=True))


def test_leading_dimensions_and_single_gradients(gpu):
    x, w, b = rand(1, 4, 5, 24).cuda(), rand(2, 12, 24).cuda(), rand(3, 12).cuda()
    y = g.linear(x, w, b, activation="silu")
    assert y.shape == (4, 5, 12) and torch.equal(y.view(20, 12), g.linear(x.view(20, 24), w, b, "silu"))
    dy = rand(4, 4, 5, 12).cuda()
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    every = torch.autograd.grad(g.linear(*leaves, activation="silu"), leaves, dy)
    for i in range(3):
        args = [t.detach().requires_grad_(j == i) for j, t in enumerate(leaves)]
        one, = torch.autograd.grad(g.linear(*args, activation="silu"), args[i], dy)
        assert torch.equal(one, every[i])


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_against_differences(gpu, dtype):
    """Directional derivatives of sum(dy * y) by differences in 64 bits of the plain form."""
    m, n, k = 40, 24, 56
    x, w, b = (rand(i, *s, dtype=dtype).double() for i, s in enumerate(((m, k), (n, k), (n,))))
    w = (w * k ** -0.5).to(dtype).double()
    dy = rand(9, m, n, dtype=dtype)
    keep = lu.mask(m, n, 0.3, 5, 1)
    f = lambda x, w, b: float((dy.double() * lu.act("gelu", x @ w.t() + b)[0] * keep).sum())
    leaves = [t.to(dtype).cuda().requires_grad_() for t in (x, w, b)]
    y = g.linear(*leaves, activation="gelu", p=0.3, seed=5, offset=1)
    grads = torch.autograd.grad(y, leaves, dy.cuda())
    _, _, z, dz = lu.linear(x.to(dtype), w.to(dtype), b.to(dtype), "gelu", keep, None, dtype)
    bounds = lu.linear_grads(dy, x, w, z, dz, "gelu", keep, dtype)
    for i, (t, grad) in enumerate(zip((x, w, b), grads)):
        step = 1e-4 * rand(20 + i, *t.shape).double()
        up, down = [x, w, b], [x, w, b]
        up[i], down[i] = t + step, t - step
        want = (f(*up) - f(*down)) / 2
        got = float((grad.double().cpu() * step).sum())
        # the gradient's own bound along the step, and the difference's third order:
        # 1e-12 of sums of at most 1e5 terms of size 10
        tol = float((bounds[i][1] * step.abs()).sum()) + 1e-6
        assert abs(got - want) <= tol, (i, got, want, tol)


# experts ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,e,k,how", [(600, 8, 2, "one"), (3000, 5, 1, "uneven"), (70, 1000, 4, "many"),
                                       (40, 32, 32, "all"), (200, 4, 2, "none")])
def test_uneven_experts(gpu, dtype, t, e, k, how):
    """All rows at one expert, empty experts, more experts than rows, every expert for
    every token, tokens that have none: forward and backward against products one by
    one in 64 bits."""
    d, n = 64, 48
    logits = rand(t, t, e)
    if how == "one":
        logits[:, 0] = 9.0
        logits[:, 1:] = -math.inf
    elif how == "uneven":
        logits += torch.linspace(0, 12, e)
    elif how == "none":
        logits[::2] = -math.inf
    r = g.route(logits.cuda(), k)
    order, offsets = r.order.cpu().long(), r.offsets.cpu().tolist()
    x, w, b = rand(1, t, d, dtype=dtype), rand(2, e, n, d, dtype=dtype, scale=d ** -0.5), rand(3, e, n, dtype=dtype)
    leaves = [v.cuda().requires_grad_() for v in (x, w, b)]
    y = g.expert_linear(leaves[0], leaves[1], r, leaves[2], gather=True)
    dy = rand(4, t * k, n, dtype=dtype)
    dx, dw, db = torch.autograd.grad(y, leaves, dy.cuda())
    live = offsets[-1]
    assert not y[live:].any()
    expert = torch.repeat_interleave(torch.arange(e), torch.tensor(offsets).diff())
    token = order[:live] // k
    xd, wd = x.double()[token], w.double()[expert]
    ref = torch.bmm(wd, xd[:, :, None])[:, :, 0] + b.double()[expert]
    err = (d + 4) * lu.V * (torch.bmm(wd.abs(), xd.abs()[:, :, None])[:, :, 0] + b.double().abs()[expert])
    lu.close(y[:live], ref, err + lu.rounding(ref.abs() + err, dtype), "y")
    g64 = dy.double()[:live]
    ref_dw, size = torch.zeros(e, n, d, dtype=torch.float64), torch.zeros(e, n, d, dtype=torch.float64)
    ref_db, size_b = torch.zeros(e, n, dtype=torch.float64), torch.zeros(e, n, dtype=torch.float64)
    for i in range(e):
        a, z = offsets[i], offsets[i + 1]
        ref_dw[i], size[i] = g64[a:z].t() @ xd[a:z], g64[a:z].abs().t() @ xd[a:z].abs()
        ref_db[i], size_b[i] = g64[a:z].sum(0), g64[a:z].abs().sum(0)
    rows = t * k + 2
    lu.close(dw, ref_dw, rows * lu.V * size + lu.rounding(ref_dw.abs() * 1.01, dtype), "dw")
    lu.close(db, ref_db, rows * lu.V * size_b + lu.rounding(ref_db.abs() * 1.01, dtype), "db")
    part = torch.bmm(g64[:, None], wd)[:, 0]
    size = torch.bmm(g64.abs()[:, None], wd.abs())[:, 0]
    ref_dx = torch.zeros(t, d, dtype=torch.float64).index_add_(0, token, part)
    err = torch.zeros(t, d, dtype=torch.float64).index_add_(0, token, (n + k + 2) * lu.V * size)
    lu.close(dx, ref_dx, err + lu.rounding(ref_dx.abs() + err, dtype), "dx")


@pytest.mark.parametrize("t", [6, 200])
def test_expert_strides(gpu, t):
    """Weights and rows that are slices of wider tensors, at odd addresses."""
    r = g.route(rand(1, t, 4).cuda(), 2)
    wide = rand(2, 4, 40, 77).cuda()
    x = rand(3, t, 80).cuda()[:, 1:66]
    w = wide[:, 2:35, 5:70]
    want = g.expert_linear(x.contiguous(), w.contiguous(), r, gather=True)
    assert torch.equal(g.expert_linear(x, w, r, gather=True), want)
    h = torch.cat((want, want), 1)[:, 3:36]
    assert torch.equal(g.combine(h, r), g.combine(h.contiguous(), r))


@pytest.mark.parametrize("t,dtype", [(5, torch.float32), (300, torch.float32), (300, torch.bfloat16)])
def test_offsets_that_begin_late(gpu, t, dtype):
    """Offsets of a caller's own that begin behind 0: the rows before the first expert's
    have no meaning, and the others are those of their experts."""
    e, d, n = 4, 24, 40
    w, b = rand(1, e, n, d, dtype=dtype).cuda(), rand(2, e, n, dtype=dtype).cuda()
    r = g.route(rand(3, t, e).cuda(), 1)
    x = rand(4, t, d, dtype=dtype).cuda()
    dy = rand(5, t, n, dtype=dtype).cuda()
    late = min(int(r.offsets[1]), 3)
    leaves = [v.clone().requires_grad_() for v in (x, w, b)]
    want = g.expert_linear(leaves[0], leaves[1], r, leaves[2], activation="silu")
    grads = torch.autograd.grad(want, leaves, dy)
    r.offsets[0] = late
    got = g.expert_linear(leaves[0], leaves[1], r, leaves[2], activation="silu")
    back = torch.autograd.grad(got, leaves, dy)
    assert torch.equal(got[late:], want[late:])
    assert torch.equal(back[0][late:], grads[0][late:])
    assert torch.equal(back[1][1:], grads[1][1:]) and torch.equal(back[2][1:], grads[2][1:])


def test_a_routing_is_made_by_route(gpu):
    r = g.route(rand(1, 6, 4).cuda(), 2)
    for lists in (r._lists[:-1], r._lists.long(), torch.stack((r._lists, r._lists), 1)[:, 0]):
        with pytest.raises(ValueError, match="made by route"):
            g.Routing(6, 4, 2, r.weights, lists)


def test_route_of_equal_rows_is_stable(gpu):
    t, e, k = 2000, 16, 4
    r = g.route(torch.zeros(t, e, device="cuda"), k)
    assert torch.equal(r.index, torch.arange(k, device="cuda", dtype=torch.int32).expand(t, k))
    rows = torch.arange(t * k, device="cuda", dtype=torch.int32).view(t, k)
    assert torch.equal(r.order, rows.t().reshape(-1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [3, 20, 150])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_activations_of_the_largest_numbers(gpu, dtype, m, name):
    """Infinities, numbers whose type's z is one, and NaN: values and slopes are the limits."""
    inf, big = math.inf, torch.finfo(dtype).max
    z = torch.tensor([inf, -inf, big, -big, math.nan, 1e4, -1e4])[torch.arange(m) % 7]
    want = torch.where(z > 0, z, torch.zeros(())).to(dtype)
    slope = (z > 0).to(dtype)
    want[z.isnan()] = slope[z.isnan()] = math.nan
    for scale in (1.0, 2.0):                # (of 2 the largest numbers' z is infinite)
        x = z.to(dtype).cuda()[:, None].requires_grad_()
        w = torch.full((9, 1), scale, dtype=dtype, device="cuda")
        y = g.linear(x, w, activation=name)
        dx, = torch.autograd.grad(y, x, torch.ones_like(y))
        assert torch.equal(y.isnan().cpu(), want.isnan()[:, None].expand(m, 9))
        there = ~want.isnan()
        assert torch.equal(y.cpu()[there], (scale * want)[there, None].expand(-1, 9))
        assert torch.equal(dx.isnan().cpu()[:, 0], want.isnan())
        # (bf16 and fp16 hold 18; 1 and 0 are exact)
        assert torch.equal(dx.cpu()[there, 0], (9 * scale * slope)[there])


# calls -----------------------------------------------------------------------

def layer(x, router, w1, w2, wo, seed):
    r = g.route(g.linear(x, router), 2)
    h = g.expert_linear(x, w1, r, activation="silu", gather=True)
    m = g.combine(g.expert_linear(h, w2, r), r, residual=x)
    return g.linear(m, wo, activation="gelu", residual=x, p=0.25, seed=seed)


def layer_inputs(seed, t=160, d=64, h=80, e=6, dtype=torch.float32):
    return [rand(seed, t, d, dtype=dtype).cuda()] + [rand(seed + i, *s, dtype=dtype, scale=d ** -0.5).cuda()
            for i, s in enumerate(((e, d), (e, h, d), (e, d, h), (d, d)), 1)]


def test_repeated_calls_are_identical(gpu):
    leaves = [v.requires_grad_() for v in layer_inputs(1, dtype=torch.bfloat16)]
    dy = rand(9, 160, 64, dtype=torch.bfloat16).cuda()
    first = None
    for _ in range(3):
        y = layer(*leaves, 7)
        out = [y.detach(), *torch.autograd.grad(y, leaves, dy)]
        if first:
            assert all(torch.equal(a, b) for a, b in zip(first, out))
        first = out


def test_two_streams(gpu):
    """Calls of different sizes on two streams at once have workspaces of their own."""
    jobs = [layer_inputs(i, t=t) for i, t in ((1, 160), (20, 700))]
    want = [layer(*v, 3) for v in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(layer(*jobs[i], 3))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(v, want[i]) for v in got[i])


def test_graph_of_a_training_step(gpu):
    """Forward and backward captured once, with a seed on the device: every replay is
    the eager result for the seed and the inputs that it finds."""
    static = layer_inputs(1)
    leaves = [v.clone().requires_grad_() for v in static]
    dy, seed = rand(9, 160, 64).cuda(), torch.tensor([11], dtype=torch.int64, device="cuda")

    def step():
        y = layer(*leaves, seed)
        return [y.detach(), *torch.autograd.grad(y, leaves, dy)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            step()                          # the stream's workspace
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step()
    seen = []
    for i in range(4):
        with torch.no_grad():
            leaves[0].copy_(rand(100 + i, 160, 64))
            seed.fill_(50 + i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        seen.append(got[0])
    assert not torch.equal(seen[0], seen[1])


def test_graphs_that_share_a_workspace(gpu):
    """Two graphs of different sizes on one stream, replayed in turn with eager calls
    between them."""
    stream = torch.cuda.Stream()
    jobs = [layer_inputs(i, t=t) for i, t in ((1, 70), (20, 700))]
    graphs, out = [], []
    with torch.cuda.stream(stream):
        want = [layer(*v, 3) for v in reversed(jobs)][::-1]
    torch.cuda.synchronize()
    for v in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            out.append(layer(*v, 3))
    with torch.cuda.stream(stream):
        for _ in range(3):
            for i in (0, 1, 1, 0):
                out[i].zero_()
                graphs[i].replay()
                layer(*jobs[1 - i], 3)
                stream.synchronize()
                assert torch.equal(out[i], want[i]), i


def test_threads_on_one_stream(gpu):
    """The launches of one call are enqueued together, whoever else calls."""
    jobs = [layer_inputs(i, t=t, d=61) for i, t in ((1, 160), (20, 700))]
    want = [layer(*v, 3) for v in jobs]
    got = [[], []]

    def work(i):
        for _ in range(10):
            got[i].append(layer(*jobs[i], 3))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 10 and all(torch.equal(v, want[i]) for v in got[i])


def test_a_routing_that_was_written_into_is_seen(gpu):
    x, w = rand(1, 6, 16).cuda().requires_grad_(), rand(2, 4, 8, 16).cuda()
    r = g.route(rand(3, 6, 4).cuda().requires_grad_(), 2)
    h = g.expert_linear(x, w, r, gather=True)
    for y in (h, g.combine(h.detach(), r), r.weights):
        r.offsets[0] = 0
        with pytest.raises(RuntimeError, match="modified by an inplace"):
            y.sum().backward(retain_graph=True)


def test_capture_that_would_need_memory_is_refused(gpu):
    # copied onto the grid: 1.3 GB, more than any test before has left to a stream
    x, w = torch.zeros(3 << 20, 101, device="cuda"), rand(2, 40, 101).cuda()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with pytest.raises(g.GettError):
        with torch.cuda.graph(graph, stream=stream):
            g.linear(x, w)
    torch.cuda.synchronize()
    assert g.linear(x[:900], w).shape == (900, 40)


def test_a_changed_seed_is_seen(gpu):
    seed = torch.tensor([1], dtype=torch.int64, device="cuda")
    x = rand(1, 8, 8).cuda().requires_grad_()
    y = g.dropout(x, 0.5, seed)
    seed.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


def test_second_derivatives_are_refused(gpu):
    x, w = rand(1, 8, 16).cuda().requires_grad_(), rand(2, 4, 16).cuda().requires_grad_()
    dx, = torch.autograd.grad(g.linear(x, w, activation="gelu").sum(), x, create_graph=True)
    assert torch.equal(dx, torch.autograd.grad(g.linear(x, w, activation="gelu").sum(), x)[0])
    with pytest.raises(RuntimeError, match="second derivatives"):
        (dx.sum() + x.sum()).backward()
    r = g.route(x, 2)
    dx, = torch.autograd.grad(r.weights.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        dx.sum().backward()


def test_no_gradients_are_kept_where_none_are_recorded(gpu):
    x, w = rand(1, 8, 16).cuda().requires_grad_(), rand(2, 4, 16).cuda()
    with torch.no_grad():
        assert not g.linear(x, w).requires_grad
    with torch.inference_mode():
        y = g.dropout(g.linear(x, w), 0.5, 1)
    assert not y.requires_grad


def test_python_refusals(gpu):
    x, w = rand(1, 6, 16).cuda(), rand(2, 8, 16).cuda()
    r = g.route(rand(3, 6, 4).cuda(), 2)
    w3 = rand(4, 4, 8, 16).cuda()
    for error, call in (
            (ValueError, lambda: g.linear(x, rand(2, 8, 15).cuda())),
            (TypeError, lambda: g.linear(x, w.half())),
            (ValueError, lambda: g.linear(x, w, rand(1, 7).cuda())),
            (TypeError, lambda: g.linear(x, w, rand(1, 8).cuda().half())),
            (TypeError, lambda: g.linear(x, w, residual=rand(1, 6, 8).cuda().half())),
            (ValueError, lambda: g.linear(x, w, residual=rand(1, 1, 8).cuda())),
            (ValueError, lambda: g.linear(x, w, p=0.5, seed=torch.tensor([1], dtype=torch.int64))),
            (ValueError, lambda: g.dropout(x, 0.5, torch.ones(2, dtype=torch.int64, device="cuda"))),
            (ValueError, lambda: g.route(x, 17)),
            (ValueError, lambda: g.route(x, 0)),
            (ValueError, lambda: g.route(x, 2, scoring="tanh")),
            (g.GettError, lambda: g.route(x, 2, groups=3)),
            (g.GettError, lambda: g.route(x, 9, groups=2, top_groups=1)),
            (TypeError, lambda: g.route(x, 2, bias=torch.zeros(16, device="cuda").half())),
            (RuntimeError, lambda: g.route(x, 2, bias=torch.zeros(16, device="cuda", requires_grad=True))),
            (ValueError, lambda: g.expert_linear(x, w3, r)),
            (ValueError, lambda: g.expert_linear(x, w3[:3], r, gather=True)),
            (TypeError, lambda: g.expert_linear(x, w3.half(), r, gather=True)),
            (ValueError, lambda: g.expert_linear(x, w3, r, rand(1, 4, 7).cuda(), gather=True)),
            (ValueError, lambda: g.combine(x, r)),
            (ValueError, lambda: g.combine(rand(1, 12, 8).cuda(), r, weights=rand(1, 6, 3).cuda())),
            (TypeError, lambda: g.combine(rand(1, 12, 8).cuda(), r, weights=r.weights.half())),
            (ValueError, lambda: g.combine(rand(1, 12, 8).cuda(), r, residual=x))):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("m,n,k", [(0, 8, 16), (3, 0, 16), (3, 8, 0), (100, 8, 0), (0, 0, 0)])
def test_empty_extents(gpu, m, n, k):
    x, w, b = (torch.zeros(s, device="cuda").requires_grad_() for s in ((m, k), (n, k), (n,)))
    with torch.no_grad():
        b.fill_(2.0)
    y = g.linear(x, w, b, activation="silu")
    assert y.shape == (m, n)
    assert torch.allclose(y, torch.nn.functional.silu(torch.full((m, n), 2.0, device="cuda")))
    dx, dw, db = torch.autograd.grad(y, (x, w, b), torch.ones_like(y))
    assert dx.shape == x.shape and not dx.any() and dw.shape == w.shape and not dw.any()
    s = torch.sigmoid(torch.tensor(2.0))
    assert torch.allclose(db, torch.full((n,), m * float(s * (1 + 2 * (1 - s))), device="cuda"))


def test_no_tokens(gpu):
    r = g.route(torch.empty(0, 4, device="cuda"), 2)
    x, w = torch.empty(0, 8, device="cuda").requires_grad_(), rand(1, 4, 6, 8).cuda().requires_grad_()
    y = g.combine(g.expert_linear(x, w, r, gather=True), r)
    assert y.shape == (0, 6)
    dx, dw = torch.autograd.grad(y, (x, w), torch.ones_like(y))
    assert dx.shape == x.shape and not dw.any()


def test_offsets_beyond_32_bits(gpu):
    """A result of 2^31 elements and more, 4.4 GB: its first and last rows."""
    m, n, k = 33000, 66000, 16
    x, w = rand(1, m, k, dtype=torch.bfloat16).cuda(), rand(2, n, k, dtype=torch.bfloat16).cuda()
    y = g.linear(x, w, p=0.5, seed=1)
    assert torch.equal(y[-5:], g.linear(x, w, p=0.5, seed=1)[-5:])
    z = g.linear(x, w)
    rows = torch.tensor([0, 1, m // 2, m - 2, m - 1])
    ref, err = linear64(x[rows].cpu(), w.cpu(), None, None, None, torch.bfloat16)
    close(z[rows], ref, err)
    kept = y[rows] != 0
    assert torch.equal(y[rows][kept], (2 * z[rows])[kept])
    d = g.dropout(z, 0.5, 1)
    assert torch.equal(d[rows], torch.where(kept, 2 * z[rows], torch.zeros_like(z[rows])))
