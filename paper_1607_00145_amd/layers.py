"""Operators of a feed-forward layer in 16 and 32 bits (include/gett_layers.h).

    y = gett.dropout(x, 0.1, seed)                       # no mask is stored
    y = gett.linear(x, w, b, activation="gelu", residual=x0, p=0.1, seed=seed)
    r = gett.route(logits, 8, scoring="sigmoid", bias=b) # eight experts a token
    h = gett.expert_linear(x, w1, r, activation="silu", gather=True)
    y = gett.combine(gett.expert_linear(h, w2, r), r)    # back to tokens

All are differentiable, backwards and once: second derivatives raise, and so do
derivatives forwards and traces (torch.jit.trace, make_fx), which would not see the
kernels.  The ``gett_*`` functions carry the names of the C interface and only
marshal arguments; the others are a convenience over torch device tensors, enqueued
on torch's current stream of the device that they lie on.
"""
from __future__ import annotations

import ctypes
import math

from . import GettError, matrix as _m

ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "silu": 3}
SCORES = {"softmax": 0, "sigmoid": 1}


class gett_dropout_t(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("seed_device", ctypes.c_void_p)]


_bound = None


def _lib():
    global _bound
    if _bound is None:
        lib = _m._lib()
        i, i64, d, p = ctypes.c_int, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p
        for name, args in (
                ("gett_dropout", [i, i64, i64, p, i64, p, p, i64, p]),
                ("gett_linear", [i, i64, i64, i64, p, i64, p, i64, p, i, p, p, i64, p, i64, p, i64,
                                 p]),
                ("gett_linear_grad", [i, i64, i64, i64, p, i64, p, i64, p, i64, p, i64, i, p, p,
                                      i64, p, i64, p, p]),
                ("gett_route", [i, i64, i, i, p, i64, i, p, i, i, i, d, p, p, p, p, p, p]),
                ("gett_route_grad", [i, i64, i, i, p, i64, i, i, d, p, p, p, i64, p]),
                ("gett_experts", [i, i64, i, i, i64, i64, p, i64, i, p, i64, i64, p, i, p, p, p,
                                  i64, p, i64, p]),
                ("gett_experts_grad", [i, i64, i, i, i64, i64, p, i64, p, i64, p, i64, i, p, i64,
                                       i64, i, p, p, p, p, i64, p, p, p]),
                ("gett_combine", [i, i64, i, i64, p, i64, i, p, p, p, i64, p, i64, p]),
                ("gett_combine_grad", [i, i64, i, i64, p, i64, p, i64, i, p, p, i, p, p, i64, p,
                                       p])):
            f = getattr(lib, name)
            f.restype, f.argtypes = i, args
        _bound = lib
    return _bound


# ----------------------------------------------------------- C interface ---
#
# Device pointers and the stream as integers (0: none); `drop` a gett_dropout_t or
# None.

def _drop_ref(drop):
    return None if drop is None else ctypes.addressof(drop)


def gett_dropout(dtype: int, rows: int, cols: int, X: int, stride_x: int, drop, Y: int,
                 stride_y: int, stream: int = 0) -> int:
    return _lib().gett_dropout(dtype, rows, cols, X or None, stride_x, _drop_ref(drop), Y or None,
                               stride_y, stream or None)


def gett_linear(dtype: int, m: int, n: int, k: int, X: int, stride_x: int, W: int, stride_w: int,
                bias: int, activation: int, drop, residual: int, stride_r: int, Z: int,
                stride_z: int, Y: int, stride_y: int, stream: int = 0) -> int:
    return _lib().gett_linear(dtype, m, n, k, X or None, stride_x, W or None, stride_w,
                              bias or None, activation, _drop_ref(drop), residual or None, stride_r,
                              Z or None, stride_z, Y or None, stride_y, stream or None)


def gett_linear_grad(dtype: int, m: int, n: int, k: int, dY: int, stride_dy: int, Z: int,
                     stride_z: int, X: int, stride_x: int, W: int, stride_w: int, activation: int,
                     drop, dX: int, stride_dx: int, dW: int, stride_dw: int, dbias: int,
                     stream: int = 0) -> int:
    return _lib().gett_linear_grad(dtype, m, n, k, dY or None, stride_dy, Z or None, stride_z,
                                   X or None, stride_x, W or None, stride_w, activation,
                                   _drop_ref(drop), dX or None, stride_dx, dW or None, stride_dw,
                                   dbias or None, stream or None)


def gett_route(dtype: int, tokens: int, experts: int, k: int, logits: int, stride: int,
               scoring: int, bias: int, groups: int, top_groups: int, renormalize: int,
               scale: float, weights: int, index: int, order: int, offsets: int, place: int,
               stream: int = 0) -> int:
    return _lib().gett_route(dtype, tokens, experts, k, logits or None, stride, scoring,
                             bias or None, groups, top_groups, renormalize, scale, weights or None,
                             index or None, order or None, offsets or None, place or None,
                             stream or None)


def gett_route_grad(dtype: int, tokens: int, experts: int, k: int, logits: int, stride: int,
                    scoring: int, renormalize: int, scale: float, index: int, dweights: int,
                    dlogits: int, stride_d: int, stream: int = 0) -> int:
    return _lib().gett_route_grad(dtype, tokens, experts, k, logits or None, stride, scoring,
                                  renormalize, scale, index or None, dweights or None,
                                  dlogits or None, stride_d, stream or None)


def gett_experts(dtype: int, tokens: int, k: int, experts: int, n: int, width: int, X: int,
                 stride_x: int, gather: int, W: int, stride_w: int, stride_we: int, bias: int,
                 activation: int, order: int, offsets: int, Z: int, stride_z: int, Y: int,
                 stride_y: int, stream: int = 0) -> int:
    return _lib().gett_experts(dtype, tokens, k, experts, n, width, X or None, stride_x, gather,
                               W or None, stride_w, stride_we, bias or None, activation,
                               order or None, offsets or None, Z or None, stride_z, Y or None,
                               stride_y, stream or None)


def gett_experts_grad(dtype: int, tokens: int, k: int, experts: int, n: int, width: int, dY: int,
                      stride_dy: int, Z: int, stride_z: int, X: int, stride_x: int, gather: int,
                      W: int, stride_w: int, stride_we: int, activation: int, order: int,
                      offsets: int, place: int, dX: int, stride_dx: int, dW: int, dbias: int,
                      stream: int = 0) -> int:
    return _lib().gett_experts_grad(dtype, tokens, k, experts, n, width, dY or None, stride_dy,
                                    Z or None, stride_z, X or None, stride_x, gather, W or None,
                                    stride_w, stride_we, activation, order or None, offsets or None,
                                    place or None, dX or None, stride_dx, dW or None, dbias or None,
                                    stream or None)


def gett_combine(dtype: int, tokens: int, k: int, cols: int, H: int, stride_h: int, dtype_w: int,
                 weights: int, place: int, residual: int, stride_r: int, Y: int, stride_y: int,
                 stream: int = 0) -> int:
    return _lib().gett_combine(dtype, tokens, k, cols, H or None, stride_h, dtype_w,
                               weights or None, place or None, residual or None, stride_r,
                               Y or None, stride_y, stream or None)


def gett_combine_grad(dtype: int, tokens: int, k: int, cols: int, dY: int, stride_dy: int, H: int,
                      stride_h: int, dtype_w: int, weights: int, place: int, experts: int,
                      offsets: int, dH: int, stride_dh: int, dweights: int,
                      stream: int = 0) -> int:
    return _lib().gett_combine_grad(dtype, tokens, k, cols, dY or None, stride_dy, H or None,
                                    stride_h, dtype_w, weights or None, place or None, experts,
                                    offsets or None, dH or None, stride_dh, dweights or None,
                                    stream or None)


# ------------------------------------------------------ torch convenience ---

_forward = _tracing = _modes = None   # as matrix.py has them


def _start():
    global _forward, _tracing, _modes
    if _m._torch is None:
        _m._start()
    _forward, _tracing, _modes = _m._forward, _m._tracing, _m._modes
    if _bound is None:
        _lib()
    return _m._torch


def _ptr(t):
    return None if t is None else t.data_ptr()


def _values(t):
    """t, or a copy where its memory holds other values than it has (torch's lazily
    negated views: imaginary parts of conjugates, and gradients of such)."""
    return t.resolve_neg() if t.is_neg() else t


def _dense(t):
    t = _values(t)
    return t if t.is_contiguous() else t.contiguous()


def _rows(name, t, dtype=None):
    """A device matrix whose columns are neighbours in memory: itself, or a copy.
    Returns it and its row stride."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    r, c = t.shape
    if t.is_contiguous() and (r > 1 or c > 1):   # (a negated view has every second number)
        return t, c
    t = _values(t)
    sr, sc = t.stride()
    if (c > 1 and sc != 1) or (r > 1 and sr < c):
        t = t.contiguous()
        sr = c
    return t, (sr if r > 1 else c)


def _vector(name, t, n, dtype):
    if tuple(t.shape) != (n,):
        raise ValueError(f"{name} must have {n} elements")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return t if n > 1 and t.is_contiguous() else _dense(t)


def _flat(name, x):
    """x as a matrix over its last dimension."""
    if not x.dim():
        raise ValueError(f"{name} must have a dimension")
    return x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), x.shape[-1])


def _activation(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {sorted(a for a in ACTIVATIONS if a)} or None"
                         ) from None


def _drop(p, seed, offset):
    """(p, seed's value, offset, seed's tensor or None) with the checks; None for
    no dropout, as p is rounded."""
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError("p must be in [0, 1]")
    if round(p * 65536) == 0:
        return None
    if seed is None:
        raise ValueError("dropout needs a seed")
    mask = (1 << 64) - 1
    if isinstance(seed, _m._torch.Tensor):
        if seed.dtype != _m._torch.int64 or seed.numel() != 1 or not seed.is_cuda:
            raise ValueError("a seed tensor is one int64 on the device")
        return p, 0, int(offset) & mask, seed
    return p, int(seed) & mask, int(offset) & mask, None


def _drop_struct(drop, seed):
    if drop is None:
        return None
    return gett_dropout_t(drop[0], drop[1], drop[2], None if seed is None else seed.data_ptr())


def _checked(st, what):
    if st != 0:
        raise GettError(st, what)


def _records(*tensors):
    if not _m._torch.is_grad_enabled():
        return False
    for t in tensors:
        if t is not None and t.requires_grad:
            return True
    return False


_functions = {}


def _function(name):
    """The autograd functions, made on the first use (torch is imported then)."""
    if not _functions:
        _make_functions()
    return _functions[name]


def _make_functions():
    torch = _m._torch

    class Refused(torch.autograd.Function):
        """The gradients as they are; differentiating them raises."""

        @staticmethod
        def forward(ctx, *values):
            return tuple(v.view_as(v) for v in values)

        @staticmethod
        def backward(ctx, *_):
            raise RuntimeError("the layers' operators have no second derivatives")

    def once(gradients):
        # Where gradients are recorded on the way back, somebody may ask for second
        # derivatives: what depends on the gradients then raises, even where the
        # gradient that came in is a constant.
        def backward(ctx, *dy):
            if _forward._current_level >= 0 or _tracing() or _modes():
                _m._eager("a gradient of the layers' operators", *dy)
            if not torch.is_grad_enabled():
                return gradients(ctx, *dy)
            with torch.no_grad():
                out = gradients(ctx, *dy)
            out = out if isinstance(out, tuple) else (out,)
            there = [i for i, v in enumerate(out) if v is not None]
            marked = Refused.apply(*(out[i].detach().requires_grad_() for i in there))
            result = list(out)
            for i, v in zip(there, marked):
                result[i] = v
            return tuple(result)
        return staticmethod(backward)

    class Dropout(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, seed, drop):
            ctx.drop = drop
            ctx.save_for_backward(seed)
            return _dropout(x, drop, seed)

        def gradients(ctx, dy):
            seed, = ctx.saved_tensors
            return _dropout(dy, ctx.drop, seed), None, None

        backward = once(gradients)

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, bias, residual, seed, activation, drop):
            need_x, need_w, need_b = ctx.needs_input_grad[:3]
            z = None
            if activation and (need_x or need_w or need_b):
                z = x.new_empty((x.shape[0], w.shape[0]))
            y = _linear(x, w, bias, residual, seed, activation, drop, z)
            ctx.activation, ctx.drop, ctx.sizes = activation, drop, (x.shape, w.shape)
            ctx.save_for_backward(x if need_w else None, w if need_x else None, z, seed)
            return y

        def gradients(ctx, dy):
            need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
            x, w, z, seed = ctx.saved_tensors
            dx = dw = db = None
            if need_x or need_w or need_b:
                dx, dw, db = _linear_grad(dy, z, x, w, seed, ctx.activation, ctx.drop, ctx.sizes,
                                          need_x, need_w, need_b)
            return dx, dw, db, dy if need_r else None, None, None, None

        backward = once(gradients)

    class Route(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, how, lists):
            ctx.how = how
            ctx.save_for_backward(logits, lists)
            return _route(logits, how, lists)

        def gradients(ctx, dweights):
            return _route_grad(*ctx.saved_tensors, dweights, ctx.how), None, None

        backward = once(gradients)

    class Experts(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, bias, routing, activation, gather):
            need_x, need_w, need_b = ctx.needs_input_grad[:3]
            z = None
            if activation and (need_x or need_w or need_b):
                z = x.new_empty((routing.tokens * routing.k, w.shape[1]))
            y = _experts(x, w, bias, routing, activation, gather, z)
            ctx.how = routing.tokens, routing.k, activation, gather, x.shape, w.shape
            ctx.save_for_backward(x if need_w else None, w if need_x else None, z, routing._lists)
            return y

        def gradients(ctx, dy):
            return (*_experts_grad(dy, *ctx.saved_tensors, ctx.how, *ctx.needs_input_grad[:3]),
                    None, None, None)

        backward = once(gradients)

    class Combine(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, weights, residual, routing):
            need_h, need_w = ctx.needs_input_grad[:2]
            ctx.how = routing.tokens, routing.k, routing.experts, h.shape, weights.dtype
            ctx.save_for_backward(h if need_w else None, weights if need_h else None,
                                  routing._lists)
            return _combine(h, weights, residual, routing)

        def gradients(ctx, dy):
            need_h, need_w, need_r = ctx.needs_input_grad[:3]
            dh = dw = None
            if need_h or need_w:
                dh, dw = _combine_grad(dy, *ctx.saved_tensors, ctx.how, need_h, need_w)
            return dh, dw, dy if need_r else None, None

        backward = once(gradients)

    _functions.update(dropout=Dropout, linear=Linear, route=Route, experts=Experts,
                      combine=Combine)


# dropout ---------------------------------------------------------------------

def _dropout(x, drop, seed):
    there = _m._elsewhere(x, seed)
    if there is not None:
        with there:
            return _dropout(x, drop, seed)
    code = _m._code(x.dtype)
    x, sx = _rows("x", x)
    r, c = x.shape
    y = x.new_empty((r, c))
    d = _drop_struct(drop, seed)
    st = _bound.gett_dropout(code, r, c, x.data_ptr(), sx, ctypes.addressof(d), y.data_ptr(), c,
                             _m._stream(x.get_device()))
    if st != 0:
        raise GettError(st, "gett_dropout")
    return y


def dropout(x, p: float, seed, offset: int = 0):
    """x / (1 - p) where a counter-based generator keeps it and 0 elsewhere.

    `p` is rounded to a multiple of 2^-16.  With p = 0 (up to 2^-17) the result is x
    itself, not a copy, as torch's own dropout returns it.  The mask is a function of
    `seed`, `offset` and a number's row (over all leading dimensions) and column: a
    call with the same seed and offset has the same mask, and the gradient makes it
    again.  `seed` is an integer, or an int64 device tensor of one element that is read
    when the kernel runs (a captured graph draws a new mask when it changes between
    replays; it must not change between a call and its gradient)."""
    if _forward is None:
        _start()
    flat = _flat("x", x)
    _m._code(x.dtype)
    _m._device("x", x)
    drop = _drop(p, seed, offset)
    if drop is None:
        return x
    if _forward._current_level >= 0 or _tracing() or _modes():
        _m._eager("dropout", flat)
    if _records(x):
        y = _function("dropout").apply(flat, drop[3], drop)
    else:
        y = _dropout(flat, drop, drop[3])
    return y if x.dim() == 2 else y.reshape(x.shape)


# linear ----------------------------------------------------------------------

def _linear(x, w, bias, residual, seed, activation, drop, z):
    there = _m._elsewhere(x, w, bias, residual, seed)
    if there is not None:
        with there:
            return _linear(x, w, bias, residual, seed, activation, drop, z)
    dtype = x.dtype
    code = _m._code(dtype)
    x, sx = _rows("x", x)
    w, sw = _rows("w", w, dtype)
    (m, k), (n, kw) = x.shape, w.shape
    if kw != k:
        raise ValueError(f"x has {k} columns, w {kw}")
    if bias is not None:
        bias = _vector("bias", bias, n, dtype)
    sr = 0
    if residual is not None:
        if tuple(residual.shape) != (m, n):
            raise ValueError("residual differs from the result in shape")
        residual, sr = _rows("residual", residual, dtype)
    y = x.new_empty((m, n))
    d = _drop_struct(drop, seed)
    st = _bound.gett_linear(code, m, n, k, x.data_ptr(), sx, w.data_ptr(), sw, _ptr(bias), activation,
                            _drop_ref(d), _ptr(residual), sr, _ptr(z), n, y.data_ptr(), n,
                            _m._stream(x.get_device()))
    if st != 0:
        raise GettError(st, "gett_linear")
    return y


def _linear_grad(dy, z, x, w, seed, activation, drop, sizes, need_x, need_w, need_b):
    there = _m._elsewhere(dy)
    if there is not None:
        with there:
            return _linear_grad(dy, z, x, w, seed, activation, drop, sizes, need_x, need_w, need_b)
    (m, k), (n, _) = sizes
    dtype = dy.dtype
    dy, sy = _rows("dy", dy)
    sx = sw = 0
    if need_w:
        x, sx = _rows("x", x)
    if need_x:
        w, sw = _rows("w", w)
    dx = dy.new_empty((m, k)) if need_x else None
    dw = dy.new_empty((n, k)) if need_w else None
    db = dy.new_empty(n) if need_b else None
    d = _drop_struct(drop, seed)
    _checked(_bound.gett_linear_grad(
        _m._code(dtype), m, n, k, dy.data_ptr(), sy, _ptr(z), n, _ptr(x) if need_w else None, sx,
        _ptr(w) if need_x else None, sw, activation, _drop_ref(d), _ptr(dx), k, _ptr(dw), k,
        _ptr(db), _m._stream(dy.get_device())), "gett_linear_grad")
    return dx, dw, db


def linear(x, w, bias=None, activation=None, residual=None, p: float = 0.0, seed=None,
           offset: int = 0):
    """residual + dropout(act(x @ w.T + bias)) over x's last dimension.

    `activation` is None, "relu", "gelu" (with erf) or "silu"; `p`, `seed` and `offset`
    are those of `dropout`.  All tensors have one type; sums and the epilogue are in
    32 bits and rounded once.  Differentiable in x, w, bias and residual: for the
    gradient x @ w.T + bias is kept where there is an activation, and no mask."""
    if _forward is None:
        _start()
    _m._code(x.dtype)
    code = _activation(activation)
    flat = _flat("x", x)
    if w.dim() != 2:
        raise ValueError("w must be a matrix")
    shape = (*x.shape[:-1], w.shape[0])
    if residual is not None:
        if tuple(residual.shape) != shape:
            raise ValueError("residual differs from the result in shape")
        residual = _flat("residual", residual)
    drop = _drop(p, seed, offset)
    seed = None if drop is None else drop[3]
    _m._device("x", x)
    _m._device("w", w)
    if _forward._current_level >= 0 or _tracing() or _modes():
        _m._eager("linear", flat, w, bias, residual)
    if _records(x, w, bias, residual):
        y = _function("linear").apply(flat, w, bias, residual, seed, code, drop)
    else:
        y = _linear(flat, w, bias, residual, seed, code, drop, None)
    return y if x.dim() == 2 else y.reshape(shape)


# routing ---------------------------------------------------------------------

class Routing:
    """The experts of `tokens` tokens, as `route` makes it.

    ``weights`` (float32, differentiable) and ``index`` (int32) are tokens x k;
    ``order`` lists the rows token * k + choice expert after expert (-1 behind the
    last), ``offsets`` says where each expert's begin, ``place`` is where `order`
    has each row (-1: nowhere).  The lists are parts of one tensor, not to be
    written into (a backward pass raises where they were)."""

    __slots__ = ("tokens", "experts", "k", "weights", "_lists")

    def __init__(self, tokens, experts, k, weights, lists):
        if (lists.dtype is not _m._torch.int32 or not lists.is_contiguous()
                or lists.numel() != 3 * tokens * k + experts + 1):
            raise ValueError("a Routing is made by route")
        self.tokens, self.experts, self.k = tokens, experts, k
        self.weights, self._lists = weights, lists   # index, order, place, offsets

    @property
    def index(self):
        t, k = self.tokens, self.k
        return self._lists.as_strided((t, k), (k, 1), 0)

    @property
    def order(self):
        n = self.tokens * self.k
        return self._lists.as_strided((n,), (1,), n)

    @property
    def place(self):
        t, k = self.tokens, self.k
        return self._lists.as_strided((t, k), (k, 1), 2 * t * k)

    @property
    def offsets(self):
        return self._lists.as_strided((self.experts + 1,), (1,), 3 * self.tokens * self.k)


def _addresses(lists, n):
    """Of a routing's index, order, place and offsets; n = tokens * k."""
    p = lists.data_ptr()
    return p, p + 4 * n, p + 8 * n, p + 12 * n


def _route(logits, how, lists):
    there = _m._elsewhere(logits, how[2])
    if there is not None:
        with there:
            return _route(logits, how, lists)
    k, scoring, bias, groups, top_groups, renormalize, scale = how
    logits, stride = _rows("logits", logits)
    t, e = logits.shape
    weights = logits.new_empty((t, k), dtype=_m._torch.float32)
    index, order, place, offsets = _addresses(lists, t * k)
    st = _bound.gett_route(_m._code(logits.dtype), t, e, k, logits.data_ptr(), stride, scoring,
                           _ptr(bias), groups, top_groups, renormalize, scale, weights.data_ptr(),
                           index, order, offsets, place, _m._stream(logits.get_device()))
    if st != 0:
        raise GettError(st, "gett_route")
    return weights


def _route_grad(logits, lists, dweights, how):
    there = _m._elsewhere(logits, dweights)
    if there is not None:
        with there:
            return _route_grad(logits, lists, dweights, how)
    k, scoring, _, _, _, renormalize, scale = how
    logits, stride = _rows("logits", logits)
    dweights = _dense(dweights)
    t, e = logits.shape
    out = logits.new_empty((t, e))
    _checked(_bound.gett_route_grad(
        _m._code(logits.dtype), t, e, k, logits.data_ptr(), stride, scoring, renormalize, scale,
        lists.data_ptr(), dweights.data_ptr(), out.data_ptr(), e, _m._stream(logits.get_device())),
        "gett_route_grad")
    return out


def route(logits, k: int, scoring: str = "softmax", bias=None, groups: int = 1,
          top_groups=None, renormalize: bool = True, scale: float = 1.0) -> Routing:
    """k experts for each row of `logits` (tokens x experts).

    Scores are the softmax or the sigmoid of the logits; `bias` (float32, one for each
    expert, no gradient) is added for the choice only; with `groups` the experts of the
    `top_groups` groups with the largest sums of two choices are open; the weights
    are the scores of the chosen, divided by their sum unless `renormalize` is false,
    times `scale`.  Ties go to the lowest index.  An expert whose logit is -inf is never
    chosen: where fewer than k are open the last indices are -1 and their weights 0."""
    if _forward is None:
        _start()
    _m._code(logits.dtype)
    if logits.dim() != 2:
        raise ValueError("logits must be a matrix (tokens x experts)")
    _m._device("logits", logits)
    if _forward._current_level >= 0 or _tracing() or _modes():
        _m._eager("route", logits, bias)
    if scoring not in SCORES:
        raise ValueError(f"scoring must be one of {sorted(SCORES)}")
    t, e = logits.shape
    k = int(k)
    if k < 1 or k > e:
        raise ValueError(f"k must be in [1, {e}]")
    if bias is not None:
        if _records(bias):
            raise RuntimeError("the bias of the choice has no gradient: detach it")
        bias = _vector("bias", bias, e, _m._torch.float32)
    how = (k, SCORES[scoring], bias, int(groups), int(groups if top_groups is None else top_groups),
           1 if renormalize else 0, float(scale))
    lists = logits.new_empty(3 * t * k + e + 1, dtype=_m._torch.int32)
    if _records(logits):
        weights = _function("route").apply(logits, how, lists)
    else:
        weights = _route(logits, how, lists)
    return Routing(t, e, k, weights, lists)


# experts ---------------------------------------------------------------------

def _weights3(w):
    """experts x n x width with neighbours along the width: itself or a copy."""
    e, n, c = w.shape
    if w.is_contiguous() and (n > 1 or c > 1):
        return w, c, n * c
    w = _values(w)
    se, sn, sc = w.stride()
    if (c > 1 and sc != 1) or (n > 1 and sn < c) or (e > 1 and se < 0):
        w = w.contiguous()
        se, sn = n * c, c
    return w, (sn if n > 1 else c), (se if e > 1 else n * c)


def _experts(x, w, bias, routing, activation, gather, z):
    there = _m._elsewhere(x, w, bias, routing._lists)
    if there is not None:
        with there:
            return _experts(x, w, bias, routing, activation, gather, z)
    t, k, e = routing.tokens, routing.k, routing.experts
    dtype = x.dtype
    x, sx = _rows("x", x)
    w, sw, se = _weights3(w)
    n, width = w.shape[1], w.shape[2]
    if bias is not None:
        bias = _dense(bias)
    y = x.new_empty((t * k, n))
    _, order, _, offsets = _addresses(routing._lists, t * k)
    st = _bound.gett_experts(_m._code(dtype), t, k, e, n, width, x.data_ptr(), sx, int(gather),
                             w.data_ptr(), sw, se, _ptr(bias), activation, order, offsets, _ptr(z), n,
                             y.data_ptr(), n, _m._stream(x.get_device()))
    if st != 0:
        raise GettError(st, "gett_experts")
    return y


def _experts_grad(dy, x, w, z, lists, how, need_x, need_w, need_b):
    there = _m._elsewhere(dy)
    if there is not None:
        with there:
            return _experts_grad(dy, x, w, z, lists, how, need_x, need_w, need_b)
    t, k, activation, gather, shape_x, shape_w = how
    e, n, width = shape_w
    dtype = dy.dtype
    dy, sy = _rows("dy", dy)
    sx = sw = se = 0
    if need_w:
        x, sx = _rows("x", x)
    if need_x:
        w, sw, se = _weights3(w)
    dx = dy.new_empty(shape_x) if need_x else None
    dw = dy.new_empty(shape_w) if need_w else None
    db = dy.new_empty((e, n)) if need_b else None
    _, order, place, offsets = _addresses(lists, t * k)
    _checked(_bound.gett_experts_grad(
        _m._code(dtype), t, k, e, n, width, dy.data_ptr(), sy, _ptr(z), n, _ptr(x), sx, int(gather),
        _ptr(w), sw, se, activation, order, offsets, place, _ptr(dx), width, _ptr(dw), _ptr(db),
        _m._stream(dy.get_device())), "gett_experts_grad")
    return dx, dw, db


def expert_linear(x, w, routing: Routing, bias=None, activation=None, gather: bool = False):
    """act(x_r @ w[e].T + bias[e]) for the rows of each expert e: tokens * k rows in the
    order of `routing`, zeros behind the last.

    With `gather` x has a row for each token (tokens x width); otherwise a row for each
    row of the result, as another `expert_linear` returns them.  `w` is experts x n x
    width, `bias` experts x n.  Differentiable in x, w and bias."""
    if _forward is None:
        _start()
    _m._code(x.dtype)
    code = _activation(activation)
    _m._device("x", x)
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError("x must be a matrix and w experts x n x width")
    rows = routing.tokens * (1 if gather else routing.k)
    if x.shape[0] != rows:
        raise ValueError(f"x has {x.shape[0]} rows, the routing {rows}")
    if w.shape[0] != routing.experts or w.shape[2] != x.shape[1]:
        raise ValueError(f"w must be {routing.experts} x n x {x.shape[1]}")
    for name, t in (("w", w), ("bias", bias)):
        if t is not None:
            if t.dtype is not x.dtype:
                raise TypeError(f"{name} is {t.dtype}, not {x.dtype}")
            _m._device(name, t)
    if bias is not None and bias.shape != w.shape[:2]:
        raise ValueError(f"bias must be {w.shape[0]} x {w.shape[1]}")
    if _forward._current_level >= 0 or _tracing() or _modes():
        _m._eager("expert_linear", x, w, bias)
    if _records(x, w, bias):
        return _function("experts").apply(x, w, bias, routing, code, bool(gather))
    return _experts(x, w, bias, routing, code, bool(gather), None)


# combine ---------------------------------------------------------------------

def _combine(h, weights, residual, routing):
    there = _m._elsewhere(h, weights, residual, routing._lists)
    if there is not None:
        with there:
            return _combine(h, weights, residual, routing)
    t, k = routing.tokens, routing.k
    dtype = h.dtype
    h, sh = _rows("h", h)
    c = h.shape[1]
    weights = _dense(weights)
    sr = 0
    if residual is not None:
        residual, sr = _rows("residual", residual, dtype)
    y = h.new_empty((t, c))
    _, _, place, _ = _addresses(routing._lists, t * k)
    st = _bound.gett_combine(_m._code(dtype), t, k, c, h.data_ptr(), sh, _m._code(weights.dtype),
                             weights.data_ptr(), place, _ptr(residual), sr, y.data_ptr(), c,
                             _m._stream(h.get_device()))
    if st != 0:
        raise GettError(st, "gett_combine")
    return y


def _combine_grad(dy, h, weights, lists, how, need_h, need_w):
    there = _m._elsewhere(dy)
    if there is not None:
        with there:
            return _combine_grad(dy, h, weights, lists, how, need_h, need_w)
    t, k, e, shape, wtype = how
    c = shape[1]
    dy, sy = _rows("dy", dy)
    sh = 0
    if need_w:
        h, sh = _rows("h", h)
    if need_h:
        weights = _dense(weights)
    dh = dy.new_empty(shape) if need_h else None
    dw = dy.new_empty((t, k), dtype=wtype) if need_w else None
    _, _, place, offsets = _addresses(lists, t * k)
    _checked(_bound.gett_combine_grad(
        _m._code(dy.dtype), t, k, c, dy.data_ptr(), sy, _ptr(h), sh, _m._code(wtype),
        _ptr(weights), place, e, offsets, _ptr(dh), c, _ptr(dw),
        _m._stream(dy.get_device())), "gett_combine_grad")
    return dh, dw


def combine(h, routing: Routing, weights=None, residual=None):
    """residual + the sum over a token's choices of weights * h, one row for each token.

    `h` has the rows of `expert_linear`; `weights` are tokens x k, in float32 or h's
    type (default: the routing's).  Differentiable in h, weights and residual."""
    if _forward is None:
        _start()
    _m._code(h.dtype)
    _m._device("h", h)
    if weights is None:
        weights = routing.weights
    t, k = routing.tokens, routing.k
    if h.dim() != 2 or h.shape[0] != t * k:
        raise ValueError(f"h must be a matrix of {t * k} rows")
    if tuple(weights.shape) != (t, k):
        raise ValueError(f"weights must be {t} x {k}")
    if weights.dtype not in (h.dtype, _m._torch.float32):
        raise TypeError(f"weights are {weights.dtype}, not float32 or {h.dtype}")
    _m._device("weights", weights)
    if residual is not None and tuple(residual.shape) != (t, h.shape[1]):
        raise ValueError("residual differs from the result in shape")
    if _forward._current_level >= 0 or _tracing() or _modes():
        _m._eager("combine", h, weights, residual)
    if _records(h, weights, residual):
        return _function("combine").apply(h, weights, residual, routing)
    return _combine(h, weights, residual, routing)
