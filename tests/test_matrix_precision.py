"""The bounds that the GPU tests hold orthogonalised matrices to, without a
GPU: numbers in two 16-bit parts keep them, numbers in one do not."""
import math

import numpy as np
import pytest

from matrix_util import bfloat16_bound, held, newton_schulz, newton_schulz_held, to_bfloat16

MUON = (3.4445, -4.7750, 2.0315)


def momentum(rng, rows, cols):
    """A few strong directions over noise, in bfloat16."""
    k = max(1, min(rows, cols) // 16)
    v = rng.standard_normal((rows, k)) @ rng.standard_normal((k, cols)) / math.sqrt(k)
    return to_bfloat16(1e-3 * (v + rng.standard_normal((rows, cols))))


def test_rounding_to_bfloat16():
    import torch
    x = np.random.default_rng(1).standard_normal(4096) * np.exp2(np.arange(4096) % 60 - 30)
    x = x.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    assert np.array_equal(to_bfloat16(x), want)
    assert np.array_equal(to_bfloat16(want), want)


def test_two_parts_hold_22_bits():
    x = np.random.default_rng(2).uniform(2.0 ** -10, 15.0, 100000)
    assert (np.abs(held(x, 2) - x) <= 2.0 ** -22 * x).all()
    assert (np.abs(held(x, 1) - x) > 2.0 ** -14 * x).any()


@pytest.mark.parametrize("shape", [(16, 16), (16, 4000), (64, 64), (130, 200), (300, 400),
                                   (517, 1000), (600, 600)])
def test_bfloat16_bound_tells_one_part_from_two(shape):
    G = momentum(np.random.default_rng(sum(shape)), *shape)
    ref = newton_schulz(G, 5, MUON, 1e-7)
    error = [np.linalg.norm(to_bfloat16(newton_schulz_held(G, 5, MUON, 1e-7, p)) - ref) /
             np.linalg.norm(ref) for p in (1, 2)]
    bound = bfloat16_bound(ref, 5)
    assert error[1] <= bound < error[0], (error, bound)
