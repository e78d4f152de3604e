"""Matrix operators for training and serving in 4 bits (include/gett_matrix.h).

    q = gett.mx_quantize(w)                    # packed along w's columns
    y = gett.mx_matmul(x, q)                   # x @ w.T, x quantised in the call
    y = gett.mx_linear(x, w)                   # the same, differentiable in x and w
    u = gett.orthogonalize(momentum)           # Newton-Schulz, for the update of w

The ``gett_*`` functions carry the names of the C interface and only marshal
arguments; the others are a convenience over torch device tensors, enqueued on
torch's current stream of the device that they lie on.
"""
from __future__ import annotations

import ctypes
import math

from . import GETT_FLOAT32, GettError, load_library

GETT_BFLOAT16 = 2
GETT_FLOAT16 = 3

_bound = None


def _lib():
    global _bound
    if _bound is None:
        lib = load_library()
        i, i64, d, p = ctypes.c_int, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p
        u64p = ctypes.POINTER(ctypes.c_uint64)
        for name, args in (
                ("gett_mx_size", [i64, i64, u64p, u64p]),
                ("gett_mx_quantize", [i, i64, i64, p, i64, i64, p, p, p, p, p]),
                ("gett_mx_dequantize", [i, i64, i64, p, p, p, i64, i64, p]),
                ("gett_mx_contract", [i64, i64, i64, d, p, p, p, p, d, i, p, i64, i64, p]),
                ("gett_mx_apply", [i64, i64, i64, d, i, p, i64, i64, p, p, d, i, p, i64, i64, p]),
                ("gett_mx_linear", [i64, i64, i64, i, p, i64, i64, i, p, i64, i64, p, i64, i64, p,
                                    p, p, p, p]),
                ("gett_mx_linear_grad", [i64, i64, i64, i, p, i64, i64, p, p, p, p, p, i64, i64, i,
                                         p, i64, i64, p]),
                ("gett_orthogonalize", [i, i64, i64, i64, p, i64, i64, i64, d, d, d, d, i, p, i64,
                                        i64, i64, p])):
            f = getattr(lib, name)
            f.restype, f.argtypes = i, args
        _bound = lib
    return _bound


# ----------------------------------------------------------- C interface ---

def gett_mx_size(rows: int, cols: int):
    """Returns (status, bytes of codes, bytes of scales)."""
    c, s = ctypes.c_uint64(), ctypes.c_uint64()
    st = _lib().gett_mx_size(rows, cols, ctypes.byref(c), ctypes.byref(s))
    return st, int(c.value), int(s.value)


def gett_mx_quantize(dtype: int, rows: int, cols: int, X: int, stride_row: int, stride_col: int,
                     codes: int, scales: int, codes_t: int, scales_t: int, stream: int = 0) -> int:
    """Device pointers and the stream as integers (0: none)."""
    return _lib().gett_mx_quantize(dtype, rows, cols, X or None, stride_row, stride_col,
                                   codes or None, scales or None, codes_t or None,
                                   scales_t or None, stream or None)


def gett_mx_dequantize(dtype: int, rows: int, cols: int, codes: int, scales: int, X: int,
                       stride_row: int, stride_col: int, stream: int = 0) -> int:
    return _lib().gett_mx_dequantize(dtype, rows, cols, codes or None, scales or None, X or None,
                                     stride_row, stride_col, stream or None)


def gett_mx_contract(m: int, n: int, k: int, alpha: float, codes_A: int, scales_A: int,
                     codes_B: int, scales_B: int, beta: float, dtype: int, C: int, stride_m: int,
                     stride_n: int, stream: int = 0) -> int:
    return _lib().gett_mx_contract(m, n, k, alpha, codes_A or None, scales_A or None,
                                   codes_B or None, scales_B or None, beta, dtype, C or None,
                                   stride_m, stride_n, stream or None)


def gett_mx_apply(m: int, n: int, k: int, alpha: float, dtype_A: int, A: int, stride_am: int,
                  stride_ak: int, codes_B: int, scales_B: int, beta: float, dtype: int, C: int,
                  stride_m: int, stride_n: int, stream: int = 0) -> int:
    return _lib().gett_mx_apply(m, n, k, alpha, dtype_A, A or None, stride_am, stride_ak,
                                codes_B or None, scales_B or None, beta, dtype, C or None,
                                stride_m, stride_n, stream or None)


def gett_orthogonalize(dtype: int, batch: int, rows: int, cols: int, G: int, stride_batch: int,
                       stride_row: int, stride_col: int, a: float, b: float, c: float, eps: float,
                       steps: int, O: int, ostride_batch: int, ostride_row: int,
                       ostride_col: int, stream: int = 0) -> int:
    return _lib().gett_orthogonalize(dtype, batch, rows, cols, G or None, stride_batch, stride_row,
                                     stride_col, a, b, c, eps, steps, O or None, ostride_batch,
                                     ostride_row, ostride_col, stream or None)


def gett_mx_linear(m: int, n: int, k: int, dtype_X: int, X: int, stride_xm: int, stride_xk: int,
                   dtype_W: int, W: int, stride_wn: int, stride_wk: int, Y: int, stride_ym: int,
                   stride_yn: int, codes_xt: int, scales_xt: int, codes_wt: int, scales_wt: int,
                   stream: int = 0) -> int:
    return _lib().gett_mx_linear(m, n, k, dtype_X, X or None, stride_xm, stride_xk, dtype_W,
                                 W or None, stride_wn, stride_wk, Y or None, stride_ym, stride_yn,
                                 codes_xt or None, scales_xt or None, codes_wt or None,
                                 scales_wt or None, stream or None)


def gett_mx_linear_grad(m: int, n: int, k: int, dtype_Y: int, dY: int, stride_ym: int,
                        stride_yn: int, codes_xt: int, scales_xt: int, codes_wt: int,
                        scales_wt: int, dX: int, stride_xm: int, stride_xk: int, dtype_W: int,
                        dW: int, stride_wn: int, stride_wk: int, stream: int = 0) -> int:
    return _lib().gett_mx_linear_grad(m, n, k, dtype_Y, dY or None, stride_ym, stride_yn,
                                      codes_xt or None, scales_xt or None, codes_wt or None,
                                      scales_wt or None, dX or None, stride_xm, stride_xk, dtype_W,
                                      dW or None, stride_wn, stride_wk, stream or None)


# ------------------------------------------------------ torch convenience ---
#
# A call is a few microseconds of host time, as long as a small matrix's
# kernel: torch is looked up once, tensors are compared as torch hands them
# out, a packed matrix is one allocation whose parts are made into tensors
# when asked for, and the C functions are called directly.

_torch = None
_current_device = _stream = None   # the current device; torch's current stream on one
_forward = _tracing = _modes = None   # torch.autograd.forward_ad; whether torch traces, has modes
_codes = {}


def _start():
    """torch and the element types' codes, on the first use."""
    global _torch, _current_device, _stream, _forward, _tracing, _modes
    import torch
    import torch.autograd.forward_ad
    c = torch._C
    _forward, _tracing, _modes = torch.autograd.forward_ad, c._is_tracing, c._len_torch_dispatch_stack
    _current_device = getattr(c, "_cuda_getDevice", torch.cuda.current_device)
    _stream = getattr(c, "_cuda_getCurrentRawStream",
                      lambda device: torch.cuda.current_stream(device).cuda_stream)
    _codes.update({torch.float32: GETT_FLOAT32, torch.bfloat16: GETT_BFLOAT16,
                   torch.float16: GETT_FLOAT16})
    _torch = torch
    _lib()


def _code(dtype) -> int:
    if _torch is None:
        _start()
    c = _codes.get(dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {dtype}: float32, bfloat16 or float16 only")
    return c


def _device(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _eager(what, *tensors):
    """Refuses what would lose a call in silence: tensors (or None) with a tangent, which
    the result would not have (a derivative of zero), and traces, which would hold
    the result's allocation and not the kernels that fill it.  Callers ask in line
    whether either may be (a call for that would be 0.2 us of a token's 7.5)."""
    for t in tensors:
        if t is not None and _forward.unpack_dual(t).tangent is not None:
            raise RuntimeError(f"{what} has no derivative forwards")
    c = _torch._C
    if _tracing() or c._get_dispatch_mode(c._TorchDispatchModeKey.PROXY) is not None:
        raise RuntimeError(f"{what} cannot be traced")


def _written(t):
    """Tells autograd that a given tensor's values have changed."""
    if not t.is_inference():
        _torch.autograd.graph.increment_version(t)


def _elsewhere(first, *others):
    """Makes current the device that all of a call's tensors (or None) lie on,
    where it is not: the call is then made again (the library launches and keeps
    its workspace on the current device).  None where it is."""
    i = first.get_device()
    for t in others:
        if t is not None and t.get_device() != i:
            raise ValueError("the tensors lie on different devices")
    return None if i == _current_device() else _torch.cuda.device(i)


def _matrix(name, t):
    """Element type code, rows, columns and strides of a device matrix."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix")
    code = _code(t.dtype)
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    (r, c), (sr, sc) = shape, t.stride()
    if sr < 1 or sc < 1 or r < 2 or c < 2:
        sr, sc = _strides(t)
    elif sc != 1 and sr != 1:
        _not_negated(t)
    return code, r, c, sr, sc


def _no_gradient(what, *tensors):
    """Refuses tensors whose gradient would be lost in silence."""
    for t in tensors:
        if t.requires_grad and _torch.is_grad_enabled():
            raise RuntimeError(f"{what} has no gradient: detach its tensors or call it under "
                               "torch.no_grad() (mx_linear with a float weight has one)")


def _not_negated(t):
    """Refuses torch's lazily negated views, whose memory holds other values than they
    have: imaginary parts of conjugates, so that no two of their numbers are
    neighbours."""
    if t.is_neg():
        raise ValueError("a lazily negated view: resolve_neg() it first")


def _strides(t):
    """(row, column) strides of the last two directions; one of extent one may
    carry any (torch leaves what it likes there, 0 included)."""
    sr, sc = t.stride()[-2:]
    r, c = t.shape[-2:]
    if (sc != 1 or c == 1) and (sr != 1 or r == 1):
        _not_negated(t)
    if r > 1 and sr < 1 or c > 1 and sc < 1:
        raise ValueError("a broadcast (zero-stride) matrix: copy it first")
    return (sr if r > 1 else max(c, 1)), (sc if c > 1 else 1)


def _sizes(rows, cols):
    t = (cols + 255) >> 8
    return rows * t * 128, t * 8 * ((rows + 15) & -16)


class MXTensor:
    """A rows x cols matrix in microscaled 4 bits, packed along its columns.

    ``codes`` and ``scales`` are uint8 device tensors of gett_mx_size's bytes."""

    __slots__ = ("rows", "cols", "_buffer", "_at", "_codes", "_scales", "_device")

    def __init__(self, rows: int, cols: int, codes, scales):
        c, s = _sizes(rows, cols)
        for name, t, n in (("codes", codes, c), ("scales", scales, s)):
            if t.numel() * t.element_size() != n or not t.is_contiguous():
                raise ValueError(f"{name} must hold {n} contiguous bytes")
            _device(name, t)
        if codes.get_device() != scales.get_device():
            raise ValueError("codes and scales lie on different devices")
        self.rows, self.cols = rows, cols
        self._buffer, self._at = (codes, scales), None
        self._codes, self._scales = codes.data_ptr(), scales.data_ptr()
        self._device = codes.get_device()

    def get_device(self):
        """The index of the device that it lies on, as a tensor's."""
        return self._device

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def device(self):
        return (self._buffer[0] if self._at is None else self._buffer).device

    @property
    def codes(self):
        if self._at is None:
            return self._buffer[0]
        return self._buffer[self._at:self._at + _sizes(self.rows, self.cols)[0]]

    @property
    def scales(self):
        if self._at is None:
            return self._buffer[1]
        c, s = _sizes(self.rows, self.cols)
        return self._buffer[self._at + c:self._at + c + s]

    def dequantize(self, dtype=None, out=None):
        """The values, as float32 unless `dtype` or `out` says otherwise."""
        r, c = self.rows, self.cols
        if _torch is None:
            _start()
        if _forward._current_level >= 0 or _tracing() or _modes():
            _eager("dequantize", out)
        i = self._device
        if out is not None or i != _current_device():
            there = _elsewhere(self, out)
            if there is not None:
                with there:
                    return self.dequantize(dtype, out)
        given = out is not None
        if not given:
            dtype = dtype or _torch.float32
            code = _code(dtype)
            out = _torch.empty((r, c), dtype=dtype, device=self.device)
            sr, sc = c or 1, 1
        else:
            if tuple(out.shape) != (r, c) or (dtype is not None and out.dtype != dtype):
                raise ValueError("out differs in shape or dtype")
            code, _, _, sr, sc = _matrix("out", out)
            _no_gradient("dequantize", out)
        st = _bound.gett_mx_dequantize(code, r, c, self._codes, self._scales, out.data_ptr(), sr, sc,
                                       _stream(i))
        if st != 0:
            raise GettError(st, "gett_mx_dequantize")
        if given:
            _written(out)
        return out


def _packed(rows, cols, device, buffer, at, codes, scales):
    """A packed matrix at byte `at` of a buffer; addresses of its parts."""
    q = MXTensor.__new__(MXTensor)
    q.rows, q.cols, q._device, q._buffer, q._at = rows, cols, device, buffer, at
    q._codes, q._scales = codes, scales
    return q


def mx_quantize(x, along: str = "cols"):
    """Pack a matrix: ``"cols"`` along its columns (x as an operand of x @ w.T),
    ``"rows"`` along its rows (its transpose as an operand), ``"both"`` in one
    pass, as a pair.  A packed matrix carries no gradient."""
    if along not in ("cols", "rows", "both"):
        raise ValueError("along must be 'cols', 'rows' or 'both'")
    code, r, c, sr, sc = _matrix("x", x)
    if _forward._current_level >= 0 or _tracing() or _modes():
        _eager("mx_quantize")
    i = x.get_device()
    if i != _current_device():
        with _elsewhere(x):
            return mx_quantize(x, along)
    # one allocation; every part a multiple of 16 bytes
    n = s = nt = sn = 0
    if along != "rows":
        n, s = _sizes(r, c)
    if along != "cols":
        nt, sn = _sizes(c, r)
    buf = _torch.empty(n + s + nt + sn, dtype=_torch.uint8, device=x.device)
    p = buf.data_ptr()
    codes = scales = codes_t = scales_t = None
    if along != "rows":
        codes, scales = p, p + n
    if along != "cols":
        codes_t = p + n + s
        scales_t = codes_t + nt
    st = _bound.gett_mx_quantize(code, r, c, x.data_ptr(), sr, sc, codes, scales, codes_t, scales_t,
                                 _stream(i))
    if st != 0:
        raise GettError(st, "gett_mx_quantize")
    if along == "cols":
        return _packed(r, c, i, buf, 0, codes, scales)
    t = _packed(c, r, i, buf, n + s, codes_t, scales_t)
    return t if along == "rows" else (_packed(r, c, i, buf, 0, codes, scales), t)


def mx_matmul(a, b, C=None, alpha: float = 1.0, beta: float = 0.0, dtype=None):
    """C <- alpha * a @ b.T + beta * C for a packed `b` (n x k) and an `a` (m x k)
    that is packed or a float matrix, which is quantised in the call.  Without C
    a new row-major one is returned, in `dtype` (default: a's, float32 for a
    packed a).  It has no gradient and refuses tensors that require one while
    gradients are recorded."""
    if not isinstance(b, MXTensor):
        raise TypeError("b must be packed (mx_quantize)")
    packed = isinstance(a, MXTensor)
    if packed:
        m, k = a.rows, a.cols
    else:
        code_a, m, k, sr, sc = _matrix("a", a)
        if a.requires_grad:
            _no_gradient("mx_matmul", a)
    n = b.rows
    if k != b.cols:
        raise ValueError(f"a has {k} columns, b {b.cols}")
    if _torch is None:
        _start()
    if _forward._current_level >= 0 or _tracing() or _modes():
        _eager("mx_matmul", None if packed else a, C)
    i = b._device
    if C is not None or not i == a.get_device() == _current_device():
        there = _elsewhere(a, b, C)
        if there is not None:
            with there:
                return mx_matmul(a, b, C, alpha, beta, dtype)
    given = C is not None
    if not given:
        if beta != 0:
            raise ValueError("beta != 0 needs C")
        if dtype is None:
            dtype = _torch.float32 if packed else a.dtype
        code, sm, sn = _code(dtype), n or 1, 1
        C = _torch.empty((m, n), dtype=dtype, device=b.device)
    else:
        if tuple(C.shape) != (m, n) or (dtype is not None and C.dtype != dtype):
            raise ValueError("C differs in shape or dtype")
        code, _, _, sm, sn = _matrix("C", C)
        _no_gradient("mx_matmul", C)
    if packed:
        st = _bound.gett_mx_contract(m, n, k, alpha, a._codes, a._scales, b._codes, b._scales, beta,
                                     code, C.data_ptr(), sm, sn, _stream(i))
    else:
        st = _bound.gett_mx_apply(m, n, k, alpha, code_a, a.data_ptr(), sr, sc, b._codes, b._scales,
                                  beta, code, C.data_ptr(), sm, sn, _stream(i))
    if st != 0:
        raise GettError(st, "gett_mx_contract" if packed else "gett_mx_apply")
    if given:
        _written(C)
    return C


def _addresses(parts, buffer):
    """Addresses of a buffer's parts; None for one that is not there."""
    if buffer is None:
        return parts
    p = buffer.data_ptr()
    return [None if at is None else p + at for at in parts]


def _linear_forward(x, w, save_x, save_w):
    """y, and what a backward pass needs of it: a buffer with the packed x^T and
    w^T that are asked for, and where in it the codes and scales of each lie."""
    cx, m, k, sxm, sxk = _matrix("x", x)
    cw, n, kw, swn, swk = _matrix("w", w)
    if kw != k:
        raise ValueError(f"x has {k} columns, w {kw}")
    there = _elsewhere(x, w)
    if there is not None:
        with there:
            return _linear_forward(x, w, save_x, save_w)
    y = _torch.empty((m, n), dtype=x.dtype, device=x.device)
    a, b = _sizes(k, m) if save_x else (0, 0)      # multiples of 16 bytes
    c, d = _sizes(k, n) if save_w else (0, 0)
    parts = ([0, a] if save_x else [None, None]) + ([a + b, a + b + c] if save_w else [None, None])
    buf = None
    if save_x or save_w:
        buf = _torch.empty(a + b + c + d, dtype=_torch.uint8, device=x.device)
    xt, xs, wt, ws = _addresses(parts, buf)
    st = _bound.gett_mx_linear(m, n, k, cx, x.data_ptr(), sxm, sxk, cw, w.data_ptr(), swn, swk,
                               y.data_ptr(), n or 1, 1, xt, xs, wt, ws, _stream(x.get_device()))
    if st != 0:
        raise GettError(st, "gett_mx_linear")
    return y, buf, parts


_function = None


def _linear_function():
    global _function
    if _function is not None:
        return _function
    torch = _torch

    class MXLinear(torch.autograd.Function):
        """y = Q(x) Q(w)^T; dx = Q(dy) Q(w^T)^T, dw = Q(dy^T) Q(x^T)^T: every
        product sums over the direction its operands are packed along, and the
        rounding's gradient is taken as one."""

        @staticmethod
        def forward(ctx, x, w):
            need_x, need_w = ctx.needs_input_grad
            y, buf, ctx.parts = _linear_forward(x, w, need_w, need_x)
            ctx.save_for_backward(buf)   # freed with the graph; hooks and checkpoints see it
            ctx.sizes = x.shape[0], w.shape[0], x.shape[1], x.dtype, w.dtype
            return y

        @staticmethod
        def backward(ctx, dy):
            # the decorated form refuses a second derivative; nobody can ask for
            # one where gradients are not recorded, and it costs 4 us of host time
            return recorded(ctx, dy) if torch.is_grad_enabled() else gradients(ctx, dy)

    def gradients(ctx, dy):
        if _forward._current_level >= 0 or _tracing() or _modes():
            _eager("a gradient of mx_linear", dy)
        need_x, need_w = ctx.needs_input_grad
        m, n, k, tx, tw = ctx.sizes
        if dy.is_neg():
            dy = dy.resolve_neg()  # (of a complex number's imaginary part)
        if dy.stride(0) < 1 or dy.stride(1) < 1:
            dy = dy.contiguous()   # the gradient of a sum is broadcast
        code, _, _, sm, sn = _matrix("dy", dy)
        buf, = ctx.saved_tensors
        xt, xs, wt, ws = _addresses(ctx.parts, buf)
        dx = torch.empty((m, k), dtype=tx, device=dy.device) if need_x else None
        dw = torch.empty((n, k), dtype=tw, device=dy.device) if need_w else None
        st = _bound.gett_mx_linear_grad(
            m, n, k, code, dy.data_ptr(), sm, sn, xt, xs, wt, ws,
            dx.data_ptr() if need_x else None, k or 1, 1, _codes[tw],
            dw.data_ptr() if need_w else None, k or 1, 1, _stream(dy.get_device()))
        if st != 0:
            raise GettError(st, "gett_mx_linear_grad")
        return dx, dw

    recorded = torch.autograd.function.once_differentiable(gradients)
    _function = MXLinear
    return _function


def mx_linear(x, w):
    """x @ w.T over the last dimension with both operands rounded to 4 bits.

    `w` is a float n x k weight (differentiable, as is `x`: gradients are
    products in 4 bits as well) or a packed one, for serving: that form keeps
    nothing that x's gradient could be formed from, and refuses an x that
    requires one while gradients are recorded."""
    shape = x.shape
    if not shape:
        raise ValueError("x must have a dimension")
    flat = x if len(shape) == 2 else x.reshape(math.prod(shape[:-1]), shape[-1])
    if isinstance(w, MXTensor):
        y = mx_matmul(flat, w)
    else:
        _code(x.dtype)
        if _forward._current_level >= 0 or _tracing() or _modes():
            _eager("mx_linear", flat, w)
        if _torch.is_grad_enabled() and (x.requires_grad or w.requires_grad):
            y = _linear_function().apply(flat, w)
        else:
            y = _linear_forward(flat, w, False, False)[0]
    return y if len(shape) == 2 else y.reshape(*shape[:-1], y.shape[1])


def orthogonalize(G, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  out=None):
    """`steps` Newton-Schulz steps X <- a X + (b S + c S^2) X, S = X X^T, from
    G / (|G| + eps), for a matrix or a stack [..., rows, cols] of them; `out`
    may be G.  It has no gradient and refuses tensors that require one while
    gradients are recorded."""
    if G.dim() < 2:
        raise ValueError("a matrix or a stack of matrices is needed")
    code = _code(G.dtype)
    _device("G", G)
    if _forward._current_level >= 0 or _tracing() or _modes():
        _eager("orthogonalize", G, out)
    there = _elsewhere(G, out)
    if there is not None:
        with there:
            return orthogonalize(G, steps, coefficients, eps, out)
    given = out is not None
    if not given:
        out = _torch.empty(G.shape, dtype=G.dtype, device=G.device)
    elif out.shape != G.shape or out.dtype != G.dtype:
        raise ValueError("out differs in shape or dtype")
    else:
        _device("out", out)
    _no_gradient("orthogonalize", G, out)
    g, o, copy = G, out, None
    if G.dim() == 2:
        g, o = G.unsqueeze(0), out.unsqueeze(0)
    elif G.dim() != 3:
        stack = (math.prod(G.shape[:-2]), *G.shape[-2:])
        g = G.reshape(stack)
        try:
            o = out.view(stack)
        except RuntimeError:   # a stack without one stride
            copy = o = _torch.empty(stack, dtype=G.dtype, device=G.device)
    n, r, c = g.shape
    if n > 1 and (g.stride(0) < 1 or o.stride(0) < 1):
        raise ValueError("a broadcast (zero-stride) stack: copy it first")
    (gr, gc), (orow, oc) = _strides(g), _strides(o)
    a, b, cc = coefficients
    st = _bound.gett_orthogonalize(code, n, r, c, g.data_ptr(), g.stride(0), gr, gc, a, b, cc, eps,
                                   int(steps), o.data_ptr(), o.stride(0), orow, oc,
                                   _stream(G.get_device()))
    if st != 0:
        raise GettError(st, "gett_orthogonalize")
    if copy is not None:
        out.copy_(copy.view(out.shape))
    elif given:
        _written(out)
    return out
