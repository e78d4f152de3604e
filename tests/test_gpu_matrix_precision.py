"""How near orthogonalised matrices are to the 64-bit ones (GPU)."""
import numpy as np
import pytest

import paper_1607_00145_amd as g
from matrix_util import bfloat16_bound, newton_schulz, newton_schulz_held
from test_matrix_precision import MUON, momentum

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(16, 16), (16, 4000), (64, 64), (130, 200), (257, 300),
                                   (300, 400), (1000, 517), (600, 600), (1100, 1210)])
def test_bfloat16_loses_no_more_than_its_rounding(gpu, shape):
    """Whatever the size, the result is the 64-bit one rounded to bfloat16
    (test_matrix_precision.py shows that iterates in one part break this bound)."""
    import torch
    G = momentum(np.random.default_rng(sum(shape)), *shape)
    dev = torch.from_numpy(G).to(torch.bfloat16).cuda()
    got = g.orthogonalize(dev).double().cpu().numpy()
    ref = newton_schulz(G, 5, MUON, 1e-7)
    error = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert error <= bfloat16_bound(ref, 5)


def newton_schulz_f32(G, steps, poly, eps):
    """In 32 bits throughout."""
    a, b, c = (np.float32(p) for p in poly)
    X = (G / (np.sqrt((G ** 2).sum()) + eps)).astype(np.float32)
    for _ in range(steps):
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X


@pytest.mark.parametrize("outlier", [1.0, 1e3, 1e5, 1e6, 1e7])
@pytest.mark.parametrize("shape", [(64, 64), (128, 2000), (512, 512)])
def test_one_element_far_above_the_rest(gpu, shape, outlier):
    """The error is that of numbers held in two parts, whose grid of 2^-36 the
    polynomial magnifies in the small numbers' directions, and of sums in 32
    bits: each emulated, and twice what the emulations err for another order of
    the sums and other roundings."""
    import torch
    rng = np.random.default_rng(1)
    G = rng.standard_normal(shape).astype(np.float32).astype(np.float64)
    G[3, 5] = outlier
    got = g.orthogonalize(torch.from_numpy(G).float().cuda()).double().cpu().numpy()
    ref = newton_schulz(G, 5, MUON, 1e-7)
    err = lambda x: np.linalg.norm(x - ref)
    held, sums = newton_schulz_held(G, 5, MUON, 1e-7, 2), newton_schulz_f32(G, 5, MUON, 1e-7)
    assert err(got) <= 2 * (err(held) + err(sums))
    # what the header says of such matrices
    said = 12 * 5 * 2.0 ** -22 * np.linalg.norm(ref) + 2.0 ** -37 * np.sqrt(G.size) * MUON[0] ** 5
    assert err(got) <= said
