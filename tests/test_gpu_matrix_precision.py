"""How near orthogonalised matrices are to the 64-bit ones (GPU)."""
import numpy as np
import pytest

import paper_1607_00145_amd as g
from matrix_util import bfloat16_bound, newton_schulz
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
