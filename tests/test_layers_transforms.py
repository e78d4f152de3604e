"""What torch may do to a call beside running it, without a GPU: derivatives forwards,
traces and lazily negated views.  The tensors are CPU tensors that claim to lie on a
device, and the library's functions a record."""
import ctypes
import os
import subprocess
import sys

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

    def resolve_neg(self):
        return torch.Tensor.resolve_neg(self).as_subclass(Claims)


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


# lazily negated views ----------------------------------------------------------

def negated(rows, cols, value=2.0):
    """-value everywhere, as torch hands out imaginary parts of conjugates: memory
    that holds `value`, its rows apart, and a mark that it is to be negated."""
    t = torch.complex(torch.zeros(rows, cols), torch.full((rows, cols), value)).conj().imag
    assert t.is_neg() and bool((t == -value).all())
    return t


def at(address, n):
    return list((ctypes.c_float * n).from_address(address))


def claims(t):
    return t.as_subclass(Claims)


# each float tensor of each call of the library: how it is made of a negated view of
# the given shape, the function, and which argument is its address
SEEN = {
    "dropout": (lambda t: g.dropout(t, 0.5, 1), (4, 1), "gett_dropout", 3),
    "linear x": (lambda t: g.linear(t, on(8, 1)), (4, 1), "gett_linear", 4),
    "linear w": (lambda t: g.linear(on(6, 1), t), (4, 1), "gett_linear", 6),
    "linear bias": (lambda t: g.linear(on(6, 16), on(1, 16), t[0]), (1, 1), "gett_linear", 8),
    "linear residual": (lambda t: g.linear(on(4, 16), on(1, 16), residual=t), (4, 1), "gett_linear", 11),
    "route": (lambda t: g.route(t, 1).weights, (4, 1), "gett_route", 4),
    "route bias": (lambda t: g.route(on(6, 1), 1, bias=t[0]), (1, 1), "gett_route", 7),
    "expert_linear x": (lambda t: g.expert_linear(t, on(3, 8, 1), routing(), gather=True), (6, 1),
                        "gett_experts", 6),
    "expert_linear w": (lambda t: g.expert_linear(on(6, 1), t[:, :, None], routing(), gather=True), (3, 1),
                        "gett_experts", 9),
    "expert_linear bias": (lambda t: g.expert_linear(on(6, 16), on(3, 1, 16), routing(), t, gather=True),
                           (3, 1), "gett_experts", 12),
    "combine h": (lambda t: g.combine(t, routing()), (12, 1), "gett_combine", 4),
    "combine weights": (lambda t: g.combine(on(1, 8), g.Routing(1, 3, 1, on(1, 1), on(7, dtype=torch.int32)),
                                            weights=t), (1, 1), "gett_combine", 7),
    "combine residual": (lambda t: g.combine(on(12, 1), routing(), residual=t), (6, 1), "gett_combine", 9),
}


@pytest.fixture
def seen(monkeypatch, calls):
    """What the functions found at their arguments' addresses when they were called."""
    found = []

    def library(where, n):
        class Library:
            def __getattr__(self, name):
                def call(*args):
                    if name == where[0]:
                        found.append(at(args[where[1]], n))
                    return 0
                return call
        for module in (layers, matrix):
            monkeypatch.setattr(module, "_bound", Library())
        return found

    return library


@pytest.mark.parametrize("name", SEEN)
def test_negated_views_are_read_as_their_values(seen, name):
    call, shape, function, argument = SEEN[name]
    found = seen((function, argument), 1)
    call(claims(negated(*shape)))
    assert found == [[-2.0]]


@pytest.mark.parametrize("name,function,argument", [
    ("dropout", "gett_dropout", 3), ("linear x", "gett_linear_grad", 4), ("linear w", "gett_linear_grad", 4),
    ("route", "gett_route_grad", 10), ("expert_linear x", "gett_experts_grad", 6),
    ("combine h", "gett_combine_grad", 4), ("combine weights", "gett_combine_grad", 4)])
def test_negated_gradients_are_read_as_their_values(seen, name, function, argument):
    """As they come out of a complex number's gradient."""
    shape = {"linear w": (1, 16), "combine weights": (6, 2)}.get(name, EVERY[name][1])
    call = {"linear x": lambda x: g.linear(x, on(1, 16)),
            "route": lambda x: g.route(x[:1], 1).weights,
            "expert_linear x": lambda x: g.expert_linear(x, on(3, 1, 16), routing(), gather=True),
            "combine h": lambda h: g.combine(h[:, :1], routing()),
            "combine weights": lambda w: g.combine(on(12, 1), routing(), weights=w),
            "dropout": lambda x: g.dropout(x[:, :1], 0.5, 1)}.get(name, EVERY[name][0])
    found = seen((function, argument), 1)
    x = on(*shape).requires_grad_()
    y = call(x)
    found.clear()
    torch.autograd.grad(y, x, claims(negated(*y.shape)))
    assert found == [[-2.0]]


def test_negated_matrices_of_the_4_bit_operators(seen):
    """Inputs and outputs are refused as broadcast ones are; a gradient is read as its values."""
    found = seen(("gett_mx_linear_grad", 4), 1)
    t = claims(negated(6, 64))
    for call in (lambda: g.mx_quantize(t), lambda: g.mx_matmul(t, packed(48, 64)),
                 lambda: g.mx_matmul(on(6, 64), packed(64, 64), t), lambda: g.mx_linear(t, on(48, 64)),
                 lambda: g.mx_linear(on(6, 64), t), lambda: g.orthogonalize(t),
                 lambda: g.orthogonalize(on(6, 64), out=t), lambda: packed(6, 64).dequantize(out=t)):
        with pytest.raises(ValueError, match="negated"):
            call()
    x = on(6, 64).requires_grad_()
    y = g.mx_linear(x, on(48, 64))
    torch.autograd.grad(y, x, claims(negated(6, 48)))
    assert found == [[-2.0]]


def test_a_call_of_the_c_interface_first():
    """It loads the library without torch, which the other calls then look up."""
    code = ("import paper_1607_00145_amd as g\n"
            "assert g.gett_dropout(7, 1, 1, 0, 1, None, 0, 1) == 1\n"
            "import torch\n"
            "for call in (lambda x: g.dropout(x, 0.5, 1), lambda x: g.linear(x, x), lambda x: g.route(x, 1)):\n"
            "    try: call(torch.zeros(4, 4))\n"
            "    except ValueError as e: assert 'device' in str(e)\n"
            "    else: assert False\n"
            "assert g.layers._forward is not None and g.layers._tracing is not None\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], check=True, cwd=root)
