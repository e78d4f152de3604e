"""Matrix operators for training and serving in 4 bits (include/gett_matrix.h).

    q = gett.mx_quantize(w)                    # packed along w's columns
    y = gett.mx_matmul(x, q)                   # x @ w.T, x quantised in the call
    y = gett.mx_linear(x, w)                   # the same, differentiable in x and w
    u = gett.orthogonalize(momentum)           # Newton-Schulz, for the update of w

The ``gett_*`` functions carry the names of the C interface and only marshal
arguments; the others are a convenience over torch device tensors, enqueued on
torch's current stream.
"""
from __future__ import annotations

import ctypes
import sys

from . import GETT_FLOAT32, GettError, load_library

_package = sys.modules[__package__]   # its _current_stream rebinds itself on the first call

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


# ------------------------------------------------------ torch convenience ---

_codes = None


def _code(dtype) -> int:
    global _codes
    if _codes is None:
        import torch
        _codes = {torch.float32: GETT_FLOAT32, torch.bfloat16: GETT_BFLOAT16,
                  torch.float16: GETT_FLOAT16}
    c = _codes.get(dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {dtype}: float32, bfloat16 or float16 only")
    return c


def _device(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _strides(t):
    """(row, column) strides of the last two directions; one of extent one may
    carry any (torch leaves what it likes there, 0 included)."""
    sr, sc = t.stride()[-2:]
    r, c = t.shape[-2:]
    if r > 1 and sr < 1 or c > 1 and sc < 1:
        raise ValueError("a broadcast (zero-stride) matrix: copy it first")
    return (sr if r > 1 else max(c, 1)), (sc if c > 1 else 1)


class MXTensor:
    """A rows x cols matrix in microscaled 4 bits, packed along its columns.

    ``codes`` and ``scales`` are uint8 device tensors of gett_mx_size's bytes."""

    __slots__ = ("rows", "cols", "codes", "scales")

    def __init__(self, rows: int, cols: int, codes, scales):
        c, s = _sizes(rows, cols)
        for name, t, n in (("codes", codes, c), ("scales", scales, s)):
            if t.numel() * t.element_size() != n or not t.is_contiguous():
                raise ValueError(f"{name} must hold {n} contiguous bytes")
            _device(name, t)
        self.rows, self.cols, self.codes, self.scales = rows, cols, codes, scales

    @property
    def shape(self):
        return (self.rows, self.cols)

    def dequantize(self, dtype=None, out=None):
        """The values, as float32 unless `dtype` or `out` says otherwise."""
        import torch
        if out is None:
            out = torch.empty((self.rows, self.cols), dtype=dtype or torch.float32,
                              device=self.codes.device)
        elif out.shape != self.shape or (dtype is not None and out.dtype != dtype):
            raise ValueError("out differs in shape or dtype")
        code = _code(out.dtype)
        _device("out", out)
        sr, sc = _strides(out)
        st = _lib().gett_mx_dequantize(code, self.rows, self.cols, self.codes.data_ptr(),
                                       self.scales.data_ptr(), out.data_ptr(), sr, sc,
                                       _package._current_stream())
        if st != 0:
            raise GettError(st, "gett_mx_dequantize")
        return out


def _sizes(rows, cols):
    t = (cols + 255) // 256
    return rows * t * 128, t * 8 * ((rows + 15) // 16 * 16)


def _packed(rows, cols, codes, scales):
    q = MXTensor.__new__(MXTensor)
    q.rows, q.cols, q.codes, q.scales = rows, cols, codes, scales
    return q


def mx_quantize(x, along: str = "cols"):
    """Pack a matrix: ``"cols"`` along its columns (x as an operand of x @ w.T),
    ``"rows"`` along its rows (its transpose as an operand), ``"both"`` in one
    pass, as a pair."""
    import torch
    if along not in ("cols", "rows", "both"):
        raise ValueError("along must be 'cols', 'rows' or 'both'")
    if x.dim() != 2:
        raise ValueError("a matrix is needed")
    code = _code(x.dtype)
    _device("x", x)
    r, c = x.shape
    sr, sc = _strides(x)
    n, s = _sizes(r, c) if along != "rows" else (0, 0)
    nt, st_ = _sizes(c, r) if along != "cols" else (0, 0)
    # one allocation; every part a multiple of 16 bytes
    buf = torch.empty(n + s + nt + st_, dtype=torch.uint8, device=x.device)
    p = buf.data_ptr()
    st = _lib().gett_mx_quantize(code, r, c, x.data_ptr(), sr, sc,
                                 p if along != "rows" else None,
                                 p + n if along != "rows" else None,
                                 p + n + s if along != "cols" else None,
                                 p + n + s + nt if along != "cols" else None, _package._current_stream())
    if st != 0:
        raise GettError(st, "gett_mx_quantize")
    out = []
    if along != "rows":
        out.append(_packed(r, c, buf[:n], buf[n:n + s]))
    if along != "cols":
        out.append(_packed(c, r, buf[n + s:n + s + nt], buf[n + s + nt:]))
    return tuple(out) if along == "both" else out[0]


def mx_matmul(a, b, C=None, alpha: float = 1.0, beta: float = 0.0, dtype=None):
    """C <- alpha * a @ b.T + beta * C for a packed `b` (n x k) and an `a` (m x k)
    that is packed or a float matrix, which is quantised in the call.  Without C
    a new row-major one is returned, in `dtype` (default: a's, float32 for a
    packed a)."""
    import torch
    if not isinstance(b, MXTensor):
        raise TypeError("b must be packed (mx_quantize)")
    packed = isinstance(a, MXTensor)
    if not packed:
        if a.dim() != 2:
            raise ValueError("a matrix is needed")
        _device("a", a)
    (m, k), n = a.shape, b.rows
    if k != b.cols:
        raise ValueError(f"a has {k} columns, b {b.cols}")
    if C is None:
        if beta != 0:
            raise ValueError("beta != 0 needs C")
        C = torch.empty((m, n), dtype=dtype or (torch.float32 if packed else a.dtype),
                        device=b.codes.device)
    elif C.shape != (m, n) or (dtype is not None and C.dtype != dtype):
        raise ValueError("C differs in shape or dtype")
    _device("C", C)
    code = _code(C.dtype)
    sm, sn = _strides(C)
    if packed:
        st = _lib().gett_mx_contract(m, n, k, alpha, a.codes.data_ptr(), a.scales.data_ptr(),
                                     b.codes.data_ptr(), b.scales.data_ptr(), beta, code,
                                     C.data_ptr(), sm, sn, _package._current_stream())
        if st != 0:
            raise GettError(st, "gett_mx_contract")
    else:
        sr, sc = _strides(a)
        st = _lib().gett_mx_apply(m, n, k, alpha, _code(a.dtype), a.data_ptr(), sr, sc,
                                  b.codes.data_ptr(), b.scales.data_ptr(), beta, code,
                                  C.data_ptr(), sm, sn, _package._current_stream())
        if st != 0:
            raise GettError(st, "gett_mx_apply")
    return C


_function = None


def _linear_function():
    global _function
    if _function is not None:
        return _function
    import torch

    class MXLinear(torch.autograd.Function):
        """y = Q(x) Q(w)^T; dx = Q(dy) Q(w^T)^T, dw = Q(dy^T) Q(x^T)^T: every
        product sums over the direction its operands are packed along, and the
        rounding's gradient is taken as one."""

        @staticmethod
        def forward(ctx, x, w):
            need_x, need_w = ctx.needs_input_grad
            xq = mx_quantize(x, "both" if need_w else "cols")
            wq = mx_quantize(w, "both" if need_x else "cols")
            xq, ctx.xt = xq if need_w else (xq, None)
            wq, ctx.wt = wq if need_x else (wq, None)
            ctx.types = x.dtype, w.dtype
            return mx_matmul(xq, wq, dtype=x.dtype)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            need_x, need_w = ctx.needs_input_grad
            if not (need_x or need_w):
                return None, None
            if dy.stride(0) < 1 or dy.stride(1) < 1:
                dy = dy.contiguous()   # the gradient of a sum is broadcast
            dq = mx_quantize(dy, "both" if need_x and need_w else "cols" if need_x else "rows")
            d, dt = dq if need_x and need_w else (dq, dq)
            dx = mx_matmul(d, ctx.wt, dtype=ctx.types[0]) if need_x else None
            dw = mx_matmul(dt, ctx.xt, dtype=ctx.types[1]) if need_w else None
            return dx, dw

    _function = MXLinear
    return _function


def mx_linear(x, w):
    """x @ w.T over the last dimension with both operands rounded to 4 bits.

    `w` is a float n x k weight (differentiable, as is `x`: gradients are
    products in 4 bits as well) or a packed one, for serving."""
    k = x.shape[-1]
    flat = x.reshape(-1, k)
    if isinstance(w, MXTensor):
        y = mx_matmul(flat, w)
    else:
        if w.dim() != 2 or w.shape[1] != k:
            raise ValueError(f"x has {k} columns, w is {tuple(w.shape)}")
        y = _linear_function().apply(flat, w)
    return y.reshape(*x.shape[:-1], y.shape[1])


def orthogonalize(G, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  out=None):
    """`steps` Newton-Schulz steps X <- a X + (b S + c S^2) X, S = X X^T, from
    G / (|G| + eps), for a matrix or a stack [..., rows, cols] of them; `out`
    may be G."""
    import torch
    if G.dim() < 2:
        raise ValueError("a matrix or a stack of matrices is needed")
    code = _code(G.dtype)
    _device("G", G)
    if out is None:
        out = torch.empty(G.shape, dtype=G.dtype, device=G.device)
    elif out.shape != G.shape or out.dtype != G.dtype:
        raise ValueError("out differs in shape or dtype")
    else:
        _device("out", out)
    g, o, copy = G, out, None
    if G.dim() != 3:
        g = G.unsqueeze(0) if G.dim() == 2 else G.reshape(-1, *G.shape[-2:])
        if G.dim() == 2:
            o = out.unsqueeze(0)
        else:
            try:
                o = out.view(-1, *out.shape[-2:])
            except RuntimeError:   # a stack without one stride
                copy = o = torch.empty(g.shape, dtype=G.dtype, device=G.device)
    n, r, c = g.shape
    if n > 1 and (g.stride(0) < 1 or o.stride(0) < 1):
        raise ValueError("a broadcast (zero-stride) stack: copy it first")
    (gr, gc), (orow, oc) = _strides(g), _strides(o)
    a, b, cc = coefficients
    st = _lib().gett_orthogonalize(code, n, r, c, g.data_ptr(), g.stride(0), gr, gc, a, b, cc, eps,
                                   int(steps), o.data_ptr(), o.stride(0), orow, oc,
                                   _package._current_stream())
    if st != 0:
        raise GettError(st, "gett_orthogonalize")
    if copy is not None:
        out.copy_(copy.view(out.shape))
    return out
