"""Which device the layers' operators run on, without a GPU: the tensors are CPU
tensors that claim to lie on a device, and the library's functions a record."""
import contextlib

import pytest
import torch

import paper_1607_00145_amd as g
from paper_1607_00145_amd import layers, matrix
from test_matrix_devices import On


@pytest.fixture
def calls(monkeypatch):
    """Records (function, device that is current) of each call; device 0 at first."""
    now, made = [0], []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                assert args[-1] == 100 + now[0]      # the stream is the device's own
                made.append((name, now[0]))
                return 0
            return call

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        yield
        now[0] = before

    layers._start()
    monkeypatch.setattr(layers, "_bound", Library())
    monkeypatch.setattr(matrix, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(matrix, "_stream", lambda index: 100 + index)
    monkeypatch.setattr(torch.cuda, "device", device)
    return made


def routing(index):
    return g.Routing(6, 3, 2, On(index, 6, 2), On(index, 3 * 12 + 4, dtype=torch.int32))


def every_call(i, j):
    """Each operator with one tensor on device i and the others on j."""
    x, w, b, y = On(i, 6, 16), On(j, 8, 16), On(j, 8), On(j, 6, 8)
    w3, h = On(j, 3, 8, 16), On(i, 12, 8)
    return [("gett_linear", lambda: g.linear(x, w)),
            ("gett_linear", lambda: g.linear(On(j, 6, 16), w, On(i, 8))),
            ("gett_linear", lambda: g.linear(On(j, 6, 16), w, b, residual=On(i, 6, 8))),
            ("gett_route", lambda: g.route(On(i, 6, 3), 2, bias=On(j, 3))),
            ("gett_experts", lambda: g.expert_linear(x, w3, routing(j), gather=True)),
            ("gett_experts", lambda: g.expert_linear(On(j, 6, 16), w3, routing(i), gather=True)),
            ("gett_combine", lambda: g.combine(h, routing(j))),
            ("gett_combine", lambda: g.combine(On(j, 12, 8), routing(j), residual=On(i, 6, 8)))]


@pytest.mark.parametrize("i,j", [(0, 1), (1, 0), (1, 2)])
def test_tensors_of_two_devices_are_refused(calls, i, j):
    for _, call in every_call(i, j):
        with pytest.raises(ValueError, match="device"):
            call()
    assert calls == []


@pytest.mark.parametrize("index", [0, 1])
def test_calls_run_on_their_tensors_device(calls, index):
    every = every_call(index, index) + [("gett_dropout", lambda: g.dropout(On(index, 6, 16), 0.5, 1))]
    for name, call in every:
        call()
        assert calls == [(name, index)]
        calls.clear()
    assert matrix._current_device() == 0
