"""The C interface of the matrix operators without a GPU: every declared
function is exported and bound, sizes of packed matrices, and the refusals,
which come before any HIP call."""
import os
import re
import subprocess

import pytest

import paper_1607_00145_amd as g

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = g.GETT_FLOAT32, g.GETT_BFLOAT16, g.GETT_FLOAT16
OK, VALUE, UNSUPPORTED = 0, 1, 3
P = 1 << 40          # an address that no call below may touch
MUON = (3.4445, -4.7750, 2.0315)


def test_every_declared_function_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "gett_matrix.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(gett_\w+)\s*\(", text)))
    assert names == ["gett_mx_apply", "gett_mx_contract", "gett_mx_dequantize", "gett_mx_linear",
                     "gett_mx_linear_grad", "gett_mx_quantize", "gett_mx_size",
                     "gett_orthogonalize"]
    out = subprocess.run(["nm", "-D", "--defined-only", g.LIB_PATH], capture_output=True,
                         text=True).stdout
    for n in names:
        assert re.search(rf"\bT {n}\b", out), n
        assert callable(getattr(g, n))


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "gett_matrix.h"\n'
                   "int main(void) { return GETT_BFLOAT16 == GETT_FLOAT32; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only",
                    "-I" + os.path.join(ROOT, "include"), str(src)], check=True)


@pytest.mark.parametrize("rows,cols,codes,scales", [
    (0, 0, 0, 0), (1, 1, 128, 128), (16, 256, 16 * 128, 128), (17, 257, 17 * 256, 2 * 8 * 32),
    (1000, 4096, 1000 * 2048, 16 * 8 * 1008)])
def test_size(rows, cols, codes, scales):
    assert g.gett_mx_size(rows, cols) == (OK, codes, scales)


def test_size_refusals():
    assert g.gett_mx_size(-1, 5)[0] == VALUE
    assert g.gett_mx_size(5, -1)[0] == VALUE
    assert g.gett_mx_size(1 << 30, 5)[0] == UNSUPPORTED
    assert g.gett_mx_size(5, 1 << 24)[0] == UNSUPPORTED


@pytest.mark.parametrize("dtype", [2, 3])
def test_the_contraction_refuses_16_bit_types(dtype):
    st, _ = g.gett_plan(dtype, "m,n", [2, 2], None, "m,k", [2, 2], None, "k,n", [2, 2], None)
    assert st == VALUE


def quantize(dtype=F32, rows=8, cols=64, X=P, sr=64, sc=1, codes=2 * P, scales=3 * P, codes_t=0,
             scales_t=0):
    return g.gett_mx_quantize(dtype, rows, cols, X, sr, sc, codes, scales, codes_t, scales_t)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=1), VALUE), (dict(dtype=9), VALUE), (dict(rows=-1), VALUE), (dict(cols=-1), VALUE),
    (dict(sr=0), VALUE), (dict(sc=0), VALUE), (dict(X=0), VALUE), (dict(X=P + 2), VALUE),
    (dict(codes=0, scales=0), VALUE), (dict(codes=0), VALUE), (dict(scales=0), VALUE),
    (dict(codes_t=4 * P), VALUE), (dict(codes=2 * P + 8), VALUE), (dict(scales=3 * P + 4), VALUE),
    (dict(codes=P), VALUE), (dict(scales=2 * P + 128), VALUE),
    (dict(codes_t=2 * P + 512, scales_t=4 * P), VALUE),
    (dict(cols=1 << 24), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED),
    (dict(rows=1 << 29, cols=1 << 23, sr=1 << 40), UNSUPPORTED),
    (dict(rows=1 << 24, codes=0, scales=0, codes_t=4 * P, scales_t=5 * P), UNSUPPORTED),
])
def test_quantize_refusals(change, status):
    assert quantize(**change) == status


def test_empty_calls_do_nothing():
    assert quantize(rows=0, X=0) == OK
    assert quantize(cols=0, X=0) == OK
    assert g.gett_mx_dequantize(F32, 0, 5, 0, 0, 0, 5, 1) == OK
    assert g.gett_mx_contract(0, 5, 3, 1.0, 0, 0, 0, 0, 0.0, F32, 0, 5, 1) == OK
    assert g.gett_mx_apply(5, 0, 3, 1.0, F32, 0, 3, 1, 0, 0, 0.0, F32, 0, 1, 1) == OK
    assert g.gett_orthogonalize(F32, 0, 5, 3, 0, 1, 3, 1, *MUON, 1e-7, 5, 0, 1, 3, 1) == OK


@pytest.mark.parametrize("change,status", [
    (dict(dtype=1), VALUE), (dict(rows=-1), VALUE), (dict(codes=0), VALUE), (dict(scales=0), VALUE),
    (dict(X=0), VALUE), (dict(X=P + 1), VALUE), (dict(sr=0), VALUE), (dict(X=2 * P), VALUE),
    (dict(X=3 * P + 64), VALUE), (dict(sr=1), UNSUPPORTED), (dict(sr=63), UNSUPPORTED),
    (dict(rows=1 << 30), UNSUPPORTED)])
def test_dequantize_refusals(change, status):
    a = dict(dtype=F32, rows=8, cols=64, codes=2 * P, scales=3 * P, X=P, sr=64, sc=1)
    a.update(change)
    assert g.gett_mx_dequantize(a["dtype"], a["rows"], a["cols"], a["codes"], a["scales"], a["X"],
                                a["sr"], a["sc"]) == status


@pytest.mark.parametrize("change,status", [
    (dict(m=-1), VALUE), (dict(k=-1), VALUE), (dict(dtype=1), VALUE), (dict(C=0), VALUE),
    (dict(C=P + 2), VALUE), (dict(sm=0), VALUE), (dict(sn=0), VALUE), (dict(ca=0), VALUE),
    (dict(sb=0), VALUE), (dict(cb=4 * P + 8), VALUE), (dict(C=2 * P), VALUE),
    (dict(C=5 * P), VALUE), (dict(sm=1), UNSUPPORTED), (dict(m=1 << 30), UNSUPPORTED),
    (dict(k=1 << 24), UNSUPPORTED)])
def test_contract_refusals(change, status):
    a = dict(m=8, n=16, k=64, dtype=F32, C=P, sm=16, sn=1, ca=2 * P, sa=3 * P, cb=4 * P, sb=5 * P)
    a.update(change)
    assert g.gett_mx_contract(a["m"], a["n"], a["k"], 1.0, a["ca"], a["sa"], a["cb"], a["sb"], 0.0,
                              a["dtype"], a["C"], a["sm"], a["sn"]) == status


@pytest.mark.parametrize("change,status", [
    (dict(ta=1), VALUE), (dict(A=0), VALUE), (dict(A=2 * P + 2), VALUE), (dict(sam=0), VALUE),
    (dict(sak=0), VALUE), (dict(cb=0), VALUE), (dict(C=2 * P), VALUE), (dict(C=4 * P), VALUE),
    (dict(sn=0), VALUE), (dict(sm=3), UNSUPPORTED), (dict(sam=1 << 60), UNSUPPORTED)])
def test_apply_refusals(change, status):
    a = dict(m=8, n=16, k=64, ta=F32, A=2 * P, sam=64, sak=1, dtype=F32, C=P, sm=16, sn=1, cb=4 * P,
             sb=5 * P)
    a.update(change)
    assert g.gett_mx_apply(a["m"], a["n"], a["k"], 1.0, a["ta"], a["A"], a["sam"], a["sak"],
                           a["cb"], a["sb"], 0.0, a["dtype"], a["C"], a["sm"], a["sn"]) == status


LINEAR = dict(m=8, n=16, k=64, tx=F32, X=P, sxm=64, sxk=1, tw=F32, W=2 * P, swn=64, swk=1, Y=3 * P,
              sym=16, syn=1, cx=4 * P, sx=5 * P, cw=6 * P, sw=7 * P)


@pytest.mark.parametrize("change,status", [
    (dict(tx=1), VALUE), (dict(tw=9), VALUE), (dict(m=-1), VALUE), (dict(k=-1), VALUE),
    (dict(X=0), VALUE), (dict(W=2 * P + 2), VALUE), (dict(Y=0), VALUE), (dict(sxm=0), VALUE),
    (dict(cx=0), VALUE), (dict(sw=0), VALUE), (dict(cw=6 * P + 8), VALUE), (dict(Y=P), VALUE),
    (dict(Y=2 * P + 64), VALUE), (dict(cx=2 * P), VALUE), (dict(cw=4 * P), VALUE),
    (dict(sw=3 * P), VALUE), (dict(sym=15), UNSUPPORTED), (dict(k=1 << 24), UNSUPPORTED),
    (dict(m=1 << 25, sxm=1 << 24, Y=1 << 62), UNSUPPORTED), (dict(m=1 << 30), UNSUPPORTED)])
def test_linear_refusals(change, status):
    a = dict(LINEAR)
    a.update(change)
    assert g.gett_mx_linear(a["m"], a["n"], a["k"], a["tx"], a["X"], a["sxm"], a["sxk"], a["tw"],
                            a["W"], a["swn"], a["swk"], a["Y"], a["sym"], a["syn"], a["cx"], a["sx"],
                            a["cw"], a["sw"]) == status


@pytest.mark.parametrize("change,status", [
    (dict(tx=1), VALUE), (dict(tw=9), VALUE), (dict(n=-1), VALUE), (dict(k=-1), VALUE),
    (dict(Y=0), VALUE), (dict(sym=0), VALUE), (dict(X=0, W=0), VALUE), (dict(X=P + 1), VALUE),
    (dict(cx=0), VALUE), (dict(cw=0), VALUE), (dict(sw=7 * P + 8), VALUE), (dict(X=3 * P), VALUE),
    (dict(W=3 * P + 32), VALUE), (dict(X=2 * P), VALUE), (dict(X=6 * P), VALUE),
    (dict(W=5 * P), VALUE), (dict(sxm=63), UNSUPPORTED), (dict(swk=2), UNSUPPORTED),
    (dict(n=1 << 24), UNSUPPORTED)])
def test_linear_grad_refusals(change, status):
    a = dict(LINEAR)
    a.update(change)
    assert g.gett_mx_linear_grad(a["m"], a["n"], a["k"], a["tx"], a["Y"], a["sym"], a["syn"],
                                 a["cx"], a["sx"], a["cw"], a["sw"], a["X"], a["sxm"], a["sxk"],
                                 a["tw"], a["W"], a["swn"], a["swk"]) == status


@pytest.mark.parametrize("change,status", [
    (dict(dtype=1), VALUE), (dict(batch=-1), VALUE), (dict(rows=-1), VALUE), (dict(steps=-1), VALUE),
    (dict(eps=-1.0), VALUE), (dict(eps=float("nan")), VALUE),
    (dict(poly=(float("inf"), 0.0, 0.0)), VALUE), (dict(poly=(1.0, float("nan"), 0.0)), VALUE),
    (dict(G=0), VALUE), (dict(O=0), VALUE), (dict(G=P + 2), VALUE), (dict(gr=0), VALUE),
    (dict(gb=0), VALUE), (dict(ob=0), VALUE), (dict(oc=0), VALUE),
    (dict(O=P + 256), VALUE), (dict(O=P, ob=1024), VALUE),
    (dict(ob=511), UNSUPPORTED), (dict(orow=63), UNSUPPORTED), (dict(steps=1001), UNSUPPORTED),
    (dict(rows=1 << 20), UNSUPPORTED), (dict(poly=(3.5, 0.0, 0.0)), UNSUPPORTED),
    (dict(poly=(1.0, -16.0, 0.0)), UNSUPPORTED), (dict(poly=(1.5, 0.5, 0.0)), UNSUPPORTED)])
def test_orthogonalize_refusals(change, status):
    a = dict(dtype=F32, batch=2, rows=8, cols=64, G=P, gb=512, gr=64, gc=1, poly=MUON, eps=1e-7,
             steps=5, O=2 * P, ob=512, orow=64, oc=1)
    a.update(change)
    assert g.gett_orthogonalize(a["dtype"], a["batch"], a["rows"], a["cols"], a["G"], a["gb"],
                                a["gr"], a["gc"], *a["poly"], a["eps"], a["steps"], a["O"], a["ob"],
                                a["orow"], a["oc"]) == status


def test_python_refusals():
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        g.mx_quantize(x)                                   # not on the device
    with pytest.raises(TypeError):
        g.mx_quantize(x.double())
    with pytest.raises(ValueError):
        g.mx_quantize(x, along="k")
    with pytest.raises(ValueError):
        g.mx_quantize(x[0])
    with pytest.raises(TypeError):
        g.mx_matmul(x, x)
    with pytest.raises(ValueError):
        g.MXTensor(4, 64, torch.zeros(3, dtype=torch.uint8), torch.zeros(128, dtype=torch.uint8))
    with pytest.raises(ValueError):
        g.orthogonalize(x[0])
    with pytest.raises(ValueError):
        g.orthogonalize(x)
    with pytest.raises(TypeError):
        g.orthogonalize(x.long())
    with pytest.raises(ValueError):
        g.mx_linear(x, torch.zeros(5, 63))
