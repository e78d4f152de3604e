"""What torch may do to a call beside running it, without a GPU: derivatives forwards,
traces and lazily negated views.  The tensors are CPU tensors that claim to lie on a
device, and the library's functions a record."""
import ctypes

import pytest
import torch
import torch.autograd.forward_ad as fwd
from torch.fx.experimental.proxy_tensor import make_fx

import paper_1607_00145_amd as g
from paper_1607_00145_amd import layers, matrix


class Claims(torch.Tensor):
    """A CPU tensor that claims to lie on device 0."""
    is_cuda = True

    def get_device(self):
        return 0


def on(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Claims)


@pytest.fixture
def calls(monkeypatch):
    """The functions of the library that were called, with their arguments."""
    made = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, args))
                return 0
            return call

    layers._start()
    for module in (layers, matrix):
        monkeypatch.setattr(module, "_bound", Library())
    monkeypatch.setattr(matrix, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(matrix, "_stream", lambda index: 0)
    monkeypatch.setattr(matrix, "_written", lambda t: None)
    return made


def routing():
    return g.Routing(6, 3, 2, on(6, 2), on(3 * 12 + 4, dtype=torch.int32))


def packed(rows, cols):
    c, s = matrix._sizes(rows, cols)
    return g.MXTensor(rows, cols, on(c, dtype=torch.uint8), on(s, dtype=torch.uint8))


# each operator as a function of one of its float tensors, and that tensor's shape
LAYERS = {
    "dropout": (lambda x: g.dropout(x, 0.5, 1), (6, 16)),
    "linear x": (lambda x: g.linear(x, on(8, 16)), (6, 16)),
    "linear w": (lambda w: g.linear(on(6, 16), w), (8, 16)),
    "linear bias": (lambda b: g.linear(on(6, 16), on(8, 16), b), (8,)),
    "linear residual": (lambda r: g.linear(on(6, 16), on(8, 16), residual=r), (6, 8)),
    "route": (lambda x: g.route(x, 2).weights, (6, 3)),
    "expert_linear x": (lambda x: g.expert_linear(x, on(3, 8, 16), routing(), gather=True), (6, 16)),
    "expert_linear w": (lambda w: g.expert_linear(on(6, 16), w, routing(), gather=True), (3, 8, 16)),
    "expert_linear bias": (lambda b: g.expert_linear(on(12, 16), on(3, 8, 16), routing(), b), (3, 8)),
    "combine h": (lambda h: g.combine(h, routing()), (12, 8)),
    "combine weights": (lambda w: g.combine(on(12, 8), routing(), weights=w), (6, 2)),
    "combine residual": (lambda r: g.combine(on(12, 8), routing(), residual=r), (6, 8)),
}
MATRIX = {
    "mx_matmul": (lambda a: g.mx_matmul(a, packed(48, 64)), (6, 64)),
    "mx_linear x": (lambda x: g.mx_linear(x, on(48, 64)), (6, 64)),
    "mx_linear w": (lambda w: g.mx_linear(on(6, 64), w), (48, 64)),
    "mx_linear packed": (lambda x: g.mx_linear(x, packed(48, 64)), (6, 64)),
    "orthogonalize": (lambda x: g.orthogonalize(x), (6, 64)),
}
EVERY = {**LAYERS, **MATRIX}


@pytest.mark.parametrize("name", EVERY)
@pytest.mark.parametrize("recorded", [True, False])
def test_derivatives_forwards_are_refused(calls, name, recorded):
    """A tensor with a tangent would come out without one: a derivative of zero."""
    call, shape = EVERY[name]
    with fwd.dual_level(), torch.set_grad_enabled(recorded):
        call(on(*shape))                  # (a level alone is nothing)
        calls.clear()
        x = fwd.make_dual(on(*shape), torch.ones(*shape).as_subclass(Claims))
        with pytest.raises(RuntimeError, match="no derivative forwards"):
            call(x)
    assert calls == []


def test_derivatives_forwards_of_outputs_are_refused(calls):
    with fwd.dual_level():
        out = fwd.make_dual(on(6, 48), torch.ones(6, 48).as_subclass(Claims))
        for call in (lambda: g.mx_matmul(on(6, 64), packed(48, 64), out),
                     lambda: g.orthogonalize(on(6, 48), out=out),
                     lambda: packed(6, 48).dequantize(out=out)):
            with pytest.raises(RuntimeError, match="no derivative forwards"):
                call()
    assert calls == []


@pytest.mark.parametrize("name", ["dropout", "linear x", "linear w", "route", "expert_linear x", "combine h",
                                  "combine weights", "mx_linear x"])
def test_derivatives_forwards_of_gradients_are_refused(calls, name):
    """Forwards over backwards: the gradient that comes in has a tangent."""
    call, shape = EVERY[name]
    x = on(*shape).requires_grad_()
    y = call(x)
    calls.clear()
    with fwd.dual_level():
        dy = fwd.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(RuntimeError, match="no derivative forwards"):
            torch.autograd.grad(y, x, dy)
    assert calls == []


@pytest.mark.parametrize("name", EVERY)
def test_traces_are_refused(calls, name):
    """A trace holds the result's allocation, and not the call that fills it."""
    call, shape = EVERY[name]
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(call, (on(*shape),), check_trace=False)
    assert calls == []
    with pytest.raises(RuntimeError, match="traced"):
        make_fx(call)(on(*shape))
    assert calls == []


def test_traces_of_packing_are_refused(calls):
    for call in (lambda x: g.mx_quantize(x).codes, lambda x: packed(6, 64).dequantize() + x):
        with pytest.raises(RuntimeError, match="traced"):
            torch.jit.trace(call, (on(6, 64),), check_trace=False)
        with pytest.raises(RuntimeError, match="traced"):
            make_fx(call)(on(6, 64))
    assert calls == []


def test_no_dropout_may_be_traced(calls):
    x = on(6, 16)
    with fwd.dual_level():
        d = fwd.make_dual(x, torch.ones(6, 16).as_subclass(Claims))
        assert g.dropout(d, 0.0, None) is d
    torch.jit.trace(lambda x: g.dropout(x, 0.0, None) + 1, (x,), check_trace=False)
    assert calls == []
