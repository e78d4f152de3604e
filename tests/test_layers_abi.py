"""The C interface of the layers' operators without a GPU: every declared function
is exported and bound, the refusals, which come before any HIP call, and the tiles
that products take."""
import ctypes
import math
import os
import re
import subprocess

import pytest

import paper_1607_00145_amd as g
from paper_1607_00145_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = g.GETT_FLOAT32, g.GETT_BFLOAT16, g.GETT_FLOAT16
OK, VALUE, UNSUPPORTED = 0, 1, 3
P = 1 << 40          # addresses that no call below may touch
Q, R, S, T = P + (1 << 34), P + (1 << 35), P + (1 << 36), P + (1 << 37)


def test_every_declared_function_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "gett_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(gett_\w+)\s*\(", text)))
    assert names == ["gett_combine", "gett_combine_grad", "gett_dropout", "gett_experts",
                     "gett_experts_grad", "gett_linear", "gett_linear_grad", "gett_route",
                     "gett_route_grad"]
    out = subprocess.run(["nm", "-D", "--defined-only", g.LIB_PATH], capture_output=True,
                         text=True).stdout
    for n in names:
        assert re.search(rf"\bT {n}\b", out), n
        assert callable(getattr(g, n))


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "gett_layers.h"\n'
                   "int main(void) { gett_dropout_t d = {0}; return (int)d.p; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only",
                    "-I" + os.path.join(ROOT, "include"), str(src)], check=True)


def drop(p, seed_device=0):
    return g.gett_dropout_t(p, 1, 2, seed_device or None)


# dropout ---------------------------------------------------------------------

@pytest.mark.parametrize("args,status", [
    ((7, 4, 8, P, 8, drop(0.5), Q, 8), VALUE),               # element type
    ((F32, -1, 8, P, 8, drop(0.5), Q, 8), VALUE),
    ((F32, 4, 8, P, 7, drop(0.5), Q, 8), VALUE),             # rows overlap
    ((F32, 4, 8, P, 8, None, Q, 8), VALUE),
    ((F32, 4, 8, P, 8, drop(-0.1), Q, 8), VALUE),
    ((F32, 4, 8, P, 8, drop(1.5), Q, 8), VALUE),
    ((F32, 4, 8, P, 8, drop(math.nan), Q, 8), VALUE),
    ((F32, 4, 8, P, 8, drop(0.5, P + 4), Q, 8), VALUE),      # a seed's alignment
    ((F32, 4, 8, 0, 8, drop(0.5), Q, 8), VALUE),
    ((F32, 4, 8, P + 2, 8, drop(0.5), Q, 8), VALUE),
    ((F32, 4, 8, P, 8, drop(0.5), P + 4, 8), VALUE),         # overlap
    ((F32, 4, 8, P, 8, drop(0.5), P, 9), VALUE),             # in place, other rows
    ((F32, 1 << 30, 8, P, 8, drop(0.5), Q, 8), UNSUPPORTED),
    ((F32, 4, 1 << 21, P, 1 << 21, drop(0.5), Q, 1 << 21), UNSUPPORTED),
    ((F32, 0, 8, 0, 8, drop(0.5), 0, 8), OK),
    ((F32, 4, 0, 0, 8, drop(0.5), 0, 8), OK)])
def test_dropout_refusals(args, status):
    assert g.gett_dropout(*args) == status


# linear ----------------------------------------------------------------------

def linear(dtype=BF16, m=4, n=8, k=16, X=P, sx=16, W=Q, sw=16, bias=0, act=0, d=None, res=0, sr=8,
           Z=0, sz=8, Y=R, sy=8):
    return g.gett_linear(dtype, m, n, k, X, sx, W, sw, bias, act, d, res, sr, Z, sz, Y, sy)


@pytest.mark.parametrize("how,status", [
    (dict(dtype=9), VALUE), (dict(act=4), VALUE), (dict(act=-1), VALUE), (dict(d=drop(2.0)), VALUE),
    (dict(m=-1), VALUE), (dict(k=-1), VALUE), (dict(sx=15), VALUE), (dict(sw=15), VALUE),
    (dict(sy=7), VALUE), (dict(X=0), VALUE), (dict(W=0), VALUE), (dict(Y=0), VALUE),
    (dict(X=P + 1), VALUE), (dict(bias=S + 1), VALUE), (dict(res=S, sr=7), VALUE),
    (dict(Z=S, sz=7), VALUE), (dict(Y=P + 2), VALUE), (dict(Y=Q + 2), VALUE), (dict(bias=R), VALUE),
    (dict(res=R + 2), VALUE), (dict(res=R, sr=9), VALUE), (dict(Z=R), VALUE), (dict(Z=P), VALUE),
    (dict(Z=S, res=S), VALUE), (dict(m=1 << 30), UNSUPPORTED), (dict(k=1 << 21, sx=1 << 21,
                                                                    sw=1 << 21), UNSUPPORTED),
    (dict(m=0, X=0, Y=0), OK), (dict(n=0, W=0, Y=0), OK)])
def test_linear_refusals(how, status):
    assert linear(**how) == status


def linear_grad(dtype=BF16, m=4, n=8, k=16, dY=P, sy=8, Z=0, sz=8, X=Q, sx=16, W=R, sw=16, act=0,
                d=None, dX=S, sdx=16, dW=T, sdw=16, db=0):
    return g.gett_linear_grad(dtype, m, n, k, dY, sy, Z, sz, X, sx, W, sw, act, d, dX, sdx, dW, sdw, db)


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(act=1), VALUE),            # an activation without its Z
    (dict(act=9), VALUE), (dict(d=drop(-1.0)), VALUE), (dict(dY=0), VALUE), (dict(X=0), VALUE),
    (dict(W=0), VALUE), (dict(sdx=15), VALUE), (dict(dX=P), VALUE), (dict(dW=S), VALUE),
    (dict(db=S + 8), VALUE), (dict(db=T + 1), VALUE), (dict(k=-1), VALUE),
    (dict(k=1 << 21, sx=1 << 21, sw=1 << 21, sdx=1 << 21, sdw=1 << 21), UNSUPPORTED),
    (dict(dX=0, dW=0, db=0), OK), (dict(m=0, dY=0, X=0, dX=0, dW=0), OK)])
def test_linear_grad_refusals(how, status):
    assert linear_grad(**how) == status


# routing ---------------------------------------------------------------------

def route(dtype=F32, t=4, e=8, k=2, logits=P, ld=8, scoring=0, bias=0, groups=1, top=1, renorm=1,
          scale=1.0, w=Q, index=Q + 4096, order=Q + 8192, offsets=Q + 12288, place=Q + 16384):
    return g.gett_route(dtype, t, e, k, logits, ld, scoring, bias, groups, top, renorm, scale, w,
                        index, order, offsets, place)


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(t=-1), VALUE), (dict(e=0), VALUE), (dict(k=0), VALUE),
    (dict(k=9), VALUE), (dict(scoring=2), VALUE), (dict(groups=3), VALUE), (dict(groups=0), VALUE),
    (dict(groups=4, top=5), VALUE), (dict(groups=4, top=0), VALUE),
    (dict(groups=8, top=1), VALUE),                          # one expert is open, two are wanted
    (dict(scale=math.nan), VALUE), (dict(ld=7), VALUE), (dict(logits=0), VALUE),
    (dict(bias=P + 2), VALUE), (dict(w=0), VALUE), (dict(index=Q + 4), VALUE),
    (dict(offsets=Q + 12289), VALUE), (dict(place=P), VALUE),
    (dict(e=1025, k=2, ld=1025), UNSUPPORTED), (dict(e=64, k=33, ld=64), UNSUPPORTED),
    (dict(t=1 << 29, k=2), UNSUPPORTED), (dict(t=1 << 30, k=1), UNSUPPORTED)])
def test_route_refusals(how, status):
    assert route(**how) == status


@pytest.mark.parametrize("args,status", [
    ((F32, 4, 8, 2, P, 8, 0, 1, 1.0, Q, R, S, 8), None),
    ((1, 4, 8, 2, P, 8, 0, 1, 1.0, Q, R, S, 8), VALUE),
    ((F32, 4, 8, 2, P, 8, 3, 1, 1.0, Q, R, S, 8), VALUE),
    ((F32, 4, 8, 2, P, 8, 0, 1, math.nan, Q, R, S, 8), VALUE),
    ((F32, 4, 8, 2, P, 8, 0, 1, 1.0, Q, R, S, 7), VALUE),
    ((F32, 4, 8, 2, P, 8, 0, 1, 1.0, Q, 0, S, 8), VALUE),
    ((F32, 4, 8, 2, P, 8, 0, 1, 1.0, Q, R, P, 8), VALUE),
    ((F32, 0, 8, 2, 0, 8, 0, 1, 1.0, 0, 0, 0, 8), OK)])
def test_route_grad_refusals(args, status):
    if status is not None:
        assert g.gett_route_grad(*args) == status


# experts ---------------------------------------------------------------------

def experts(dtype=BF16, t=4, k=2, e=3, n=8, width=16, X=P, sx=16, gather=1, W=Q, sw=16, swe=128,
            bias=0, act=0, order=R, offsets=R + 4096, Z=0, sz=8, Y=S, sy=8):
    return g.gett_experts(dtype, t, k, e, n, width, X, sx, gather, W, sw, swe, bias, act, order,
                          offsets, Z, sz, Y, sy)


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(t=-1), VALUE), (dict(k=0), VALUE), (dict(e=0), VALUE),
    (dict(act=4), VALUE), (dict(X=0), VALUE), (dict(W=0), VALUE), (dict(swe=-1), VALUE),
    (dict(order=0), VALUE), (dict(offsets=0), VALUE), (dict(Y=0), VALUE), (dict(Y=P), VALUE),
    (dict(Y=Q + 256), VALUE), (dict(Y=R), VALUE), (dict(Z=S), VALUE), (dict(bias=Q + 1), VALUE),
    (dict(e=1025), UNSUPPORTED), (dict(k=33), UNSUPPORTED), (dict(t=1 << 29), UNSUPPORTED),
    (dict(t=0, X=0, Y=0, order=0, offsets=0), OK)])
def test_experts_refusals(how, status):
    assert experts(**how) == status


def experts_grad(dtype=BF16, t=4, k=2, e=3, n=8, width=16, dY=P, sy=8, Z=0, sz=8, X=Q, sx=16,
                 gather=1, W=R, sw=16, swe=128, act=0, order=S, offsets=S + 4096, place=S + 8192,
                 dX=T, sdx=16, dW=T + 4096, db=T + 8192):
    return g.gett_experts_grad(dtype, t, k, e, n, width, dY, sy, Z, sz, X, sx, gather, W, sw, swe,
                               act, order, offsets, place, dX, sdx, dW, db)


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(act=2), VALUE), (dict(act=-1), VALUE), (dict(dY=0), VALUE),
    (dict(X=0), VALUE), (dict(W=0), VALUE), (dict(order=0), VALUE), (dict(place=0), VALUE),
    (dict(offsets=0), VALUE), (dict(dX=P), VALUE), (dict(dW=T), VALUE), (dict(db=T + 4097), VALUE),
    (dict(width=-1), VALUE), (dict(width=1 << 21, sx=1 << 21, sw=1 << 21, sdx=1 << 21), UNSUPPORTED),
    (dict(dX=0, dW=0, db=0), OK)])
def test_experts_grad_refusals(how, status):
    assert experts_grad(**how) == status


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(tw=F16), VALUE), (dict(H=0), VALUE), (dict(w=0), VALUE),
    (dict(place=0), VALUE), (dict(Y=P), VALUE), (dict(res=T + 2), VALUE), (dict(sy=7), VALUE),
    (dict(t=0, H=0, w=0, place=0, Y=0), OK), (dict(c=0, H=0, w=0, place=0, Y=0), OK)])
def test_combine_refusals(how, status):
    a = dict(dtype=BF16, t=4, k=2, c=8, H=P, sh=8, tw=F32, w=Q, place=R, res=0, sr=8, Y=T, sy=8)
    a.update(how)
    assert g.gett_combine(*a.values()) == status


@pytest.mark.parametrize("how,status", [
    (dict(dtype=1), VALUE), (dict(tw=F16), VALUE), (dict(dY=0), VALUE), (dict(H=0), VALUE),
    (dict(w=0), VALUE), (dict(place=0), VALUE), (dict(offsets=0), VALUE), (dict(e=0), VALUE),
    (dict(dH=P), VALUE), (dict(dw=T), VALUE), (dict(dH=0, dw=0), OK)])
def test_combine_grad_refusals(how, status):
    a = dict(dtype=BF16, t=4, k=2, c=8, dY=P, sy=8, H=Q, sh=8, tw=F32, w=R, place=S, e=3,
             offsets=S + 4096, dH=T, sdh=8, dw=T + 4096)
    a.update(how)
    assert g.gett_combine_grad(*a.values()) == status


# tiles -----------------------------------------------------------------------

class Tiles(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("edge", "slices", "shared", "workgroups")]


def product_tiles(dtype, m, n, k):
    t = Tiles()
    f = g.load_library().gett_product_tiles
    f.argtypes, f.restype = [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_void_p], None
    f(dtype, m, n, k, ctypes.byref(t))
    return t


@pytest.mark.parametrize("dtype,m,n,k,edge", [
    (BF16, 8192, 8192, 4096, 256), (BF16, 1024, 4096, 4096, 128), (BF16, 200, 4096, 4096, 64),
    (BF16, 64, 4096, 4096, 32), (BF16, 3, 512, 4096, 32), (BF16, 2, 512, 4096, 0), (BF16, 1, 8192, 4096, 32),
    (F32, 8192, 8192, 4096, 128), (F32, 32, 512, 4096, 64), (F32, 65, 128, 64, 32), (F32, 5, 128, 64, 32),
    (F32, 4, 512, 4096, 0)])
def test_tiles_by_size(dtype, m, n, k, edge):
    assert product_tiles(dtype, m, n, k).edge == edge


def test_no_tiles_of_256_in_32_bits():
    for k in (0, 1, 64, 4096):
        for m in (65, 100, 8192, 100000):
            assert product_tiles(F32, m, m, k).edge in (32, 64, 128)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_of_any_size_fit_a_launch(dtype):
    """Blocks of 32 x 32 are workgroups of their own: no more than a launch has threads for."""
    for m in (1 << 20, (1 << 27) + 5, (1 << 30) - 1):
        for n, k in ((1, 1), (16, 16), (33, 64)):
            t = product_tiles(dtype, m, n, k)
            assert t.edge > 32 or t.workgroups <= 1 << 22, (m, n, k)


@pytest.mark.parametrize("m,n,k", [(65, 4096, 4096), (1023, 515, 1000), (300, 300, 8192), (2100, 2100, 4096)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_tiles_fit_their_counters(dtype, m, n, k):
    t = product_tiles(dtype, m, n, k)
    tiles = -(-m // t.edge) * -(-n // t.edge)
    assert t.workgroups == tiles - t.shared + t.shared * t.slices
    assert 1 <= t.slices <= 16 and 0 <= t.shared <= tiles


# Python ----------------------------------------------------------------------

def test_python_refusals_without_a_device():
    import torch
    x, w = torch.zeros(4, 16), torch.zeros(8, 16)
    with pytest.raises(ValueError, match="device"):
        g.dropout(x, 0.5, 1)
    with pytest.raises(ValueError, match="device"):
        g.linear(x, w)
    with pytest.raises(ValueError, match="device"):
        g.route(x, 2)
    with pytest.raises(TypeError, match="float64"):
        g.linear(x.double(), w.double())
    with pytest.raises(ValueError, match="activation"):
        g.linear(x, w, activation="tanh")
    with pytest.raises(ValueError, match="seed"):
        g.linear(x, w, p=0.1)
    with pytest.raises(ValueError, match="p must"):
        g.linear(x, w, p=1.1, seed=1)
    with pytest.raises(ValueError, match="residual"):
        g.linear(x, w, residual=torch.zeros(4, 9))
    with pytest.raises(ValueError, match="matrix"):
        g.linear(x, w[0])


def test_seeds_of_any_size():
    layers._start()
    assert layers._drop(0.5, -1, -2) == (0.5, (1 << 64) - 1, (1 << 64) - 2, None)
    assert layers._drop(0.0, None, 0) is None
