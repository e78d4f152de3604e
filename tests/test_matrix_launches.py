"""Calls with more workgroups than a launch may have (2^32 threads) are refused
as not supported before any HIP call (no GPU)."""
import pytest

import paper_1607_00145_amd as g
from test_matrix_abi import F32, MUON, P, UNSUPPORTED

BF16 = g.GETT_BFLOAT16


def test_quantize():
    # 32 rows a workgroup of 256 threads: 2^29 rows are 2^32 threads
    assert g.gett_mx_quantize(BF16, 1 << 29, 1, P, 1, 1, 2 * P, 3 * P, 0, 0) == UNSUPPORTED
    # 128 x 128 a workgroup, and two of them for the 256 rows that one is padded to
    n = (1 << 30) - 1
    assert g.gett_mx_quantize(BF16, 1, n, P, n, 1, 0, 0, 2 * P, 3 * P) == UNSUPPORTED


def test_dequantize():
    assert g.gett_mx_dequantize(BF16, 1 << 29, 1, 2 * P, 3 * P, P, 1, 1) == UNSUPPORTED


@pytest.mark.parametrize("m", [1, 20])
def test_products_of_few_rows(m):
    # 32 rows of B a workgroup of 512 threads
    n = 1 << 28
    assert g.gett_mx_apply(m, n, 4, 1.0, BF16, 4 * P, 4, 1, 2 * P, 3 * P, 0.0, BF16, P, n,
                           1) == UNSUPPORTED
    assert g.gett_mx_contract(m, n, 4, 1.0, 4 * P, 5 * P, 2 * P, 3 * P, 0.0, BF16, P, n,
                              1) == UNSUPPORTED


def test_products_in_tiles():
    n = 1 << 20            # 2^24 tiles of 256 x 256 and 512 threads
    assert g.gett_mx_contract(n, n, 4, 1.0, 4 * P, 5 * P, 2 * P, 3 * P, 0.0, BF16, 1 << 50,
                              n, 1) == UNSUPPORTED


@pytest.mark.parametrize("batch,rows,cols,steps", [
    (1 << 23, 16, 16, 5),          # one workgroup of 512 threads each
    (1 << 16, 300, 300, 5),        # 25 tiles at the start, 300 rows for the norm
    (1 << 16, 300, 300, 0),
    (1, 1 << 19, 1 << 19, 1)])
def test_orthogonalize(batch, rows, cols, steps):
    n = rows * cols
    assert g.gett_orthogonalize(F32, batch, rows, cols, P, n, cols, 1, *MUON, 1e-7, steps, 1 << 50,
                                n, cols, 1) == UNSUPPORTED
