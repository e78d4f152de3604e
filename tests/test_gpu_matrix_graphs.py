"""Captured matrix operators beside later calls on the same stream (GPU): a call
that needs a larger workspace leaves graphs captured before what they point at
(test_workspace_graphs.py shows the same of the addresses, without a GPU)."""
import json

import numpy as np
import pytest

import paper_1607_00145_amd as g

pytestmark = pytest.mark.gpu


def capture(stream, step):
    """`step` once eagerly (it makes the workspace), then captured."""
    import torch
    step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = step()
    return graph, outs


def replays_equal(stream, graph, outs, step, inputs, times=4):
    """New inputs, an eager step and a replay: equal outputs each time."""
    import torch
    for i in range(times):
        for t in inputs:
            t.copy_(torch.randn(t.shape, device="cuda"))
        want = [t.clone() for t in step()]
        stream.synchronize()
        graph.replay()
        stream.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), i


def test_graphs_outlive_larger_calls_on_their_stream(gpu):
    """Batches of growing size, each captured after its eager call; then every
    graph is replayed."""
    import torch
    s = torch.cuda.Stream()
    w = torch.randn(700, 900, device="cuda")
    wq = g.mx_quantize(w)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graphs = []
        for rows in (33, 400, 3000):
            x = torch.randn(rows, 900, device="cuda")
            step = lambda x=x, n=200 + rows // 4: (g.mx_matmul(x, wq), g.orthogonalize(x[:, :n]))
            graphs.append((x, step) + capture(s, step))
        for x, step, graph, outs in graphs:
            replays_equal(s, graph, outs, step, [x])
        for x, step, graph, outs in reversed(graphs):
            replays_equal(s, graph, outs, step, [x], 2)


def test_a_captured_contraction_outlives_a_matrix_operator(gpu, monkeypatch):
    """Partial tiles of K slices in the workspace that a larger call replaces."""
    import torch
    monkeypatch.setenv("GETT_FORCE_KSLICES", "8")
    gen = torch.Generator(device="cpu").manual_seed(3)
    a, b = (torch.randint(-4, 5, shape, generator=gen).float().cuda() for shape in
            ((130, 900), (900, 170)))
    c = torch.zeros(130, 170, device="cuda")
    plan = g.Plan("C[i,j] = A[i,k] * B[k,j]", C=c, A=a, B=b)
    d = json.loads(json.dumps(plan.describe()))
    assert d["kslices"] > 1 and d["partials"] == "workspace"
    want = a @ b
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph, _ = capture(s, lambda: plan(a, b, c))
        G = torch.randn(1500, 1600, device="cuda")
        O = g.orthogonalize(G)
        for _ in range(4):
            c.fill_(7.0)
            g.orthogonalize(G, out=O)
            s.synchronize()
            graph.replay()
            s.synchronize()
            assert torch.equal(c, want)
        big = g.orthogonalize(torch.randn(2600, 2500, device="cuda"))
        c.fill_(7.0)
        graph.replay()
        s.synchronize()
        assert torch.equal(c, want) and torch.isfinite(big).all()


def test_a_training_step_in_a_graph(gpu):
    """mx_linear forward and backward, captured and replayed with new inputs."""
    import torch
    s = torch.cuda.Stream()
    x = torch.randn(300, 260, device="cuda", requires_grad=True)
    w = torch.randn(200, 260, device="cuda", requires_grad=True)
    dy = torch.randn(300, 200, device="cuda")

    def step():
        y = g.mx_linear(x, w)
        return (y.detach(), *torch.autograd.grad(y, (x, w), dy))

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph, outs = capture(s, step)
        replays_equal(s, graph, outs, step, [x.detach(), w.detach(), dy])


def test_growth_inside_a_capture_is_refused(gpu):
    """A call that needs more than any before it: refused while the stream
    captures, with nothing enqueued and the capture still valid."""
    import torch
    s = torch.cuda.Stream()
    G = torch.randn(9000, 9000, device="cuda")
    O, mark = torch.full_like(G, 5.0), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        mark.add_(1.0)
        with pytest.raises(g.GettError) as e:
            g.orthogonalize(G, steps=0, out=O)
    assert e.value.status == g.GETT_ERROR_NOT_SUPPORTED
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (mark == i + 1).all() and (O == 5.0).all()
    with torch.cuda.stream(s):
        g.orthogonalize(G, steps=0, out=O)
    s.synchronize()
    want = G.double() / torch.linalg.vector_norm(G.double())
    # two parts of 2^12 x: 2^-22 of a number, or half a step of 2^-36
    assert ((O.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -37).all()
