"""Plain 64-bit forms of the matrix operators, for their tests: written from
the definitions in include/gett_matrix.h, on the CPU, sharing nothing with the
library."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_to_grid(q):
    """Nearest of GRID with q's sign; a tie goes to the even code."""
    a = np.minimum(np.abs(q), 6.0)
    d = np.abs(a[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    tied = d == best
    even = np.arange(8) % 2 == 0
    code = np.where((tied & even).any(-1), np.argmax(tied & even, -1), np.argmax(tied, -1))
    return np.where(np.signbit(q), -1.0, 1.0) * GRID[code]


def mx_values(x):
    """[rows, cols] -> the values of its packing along the columns."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    g = np.zeros((rows, blocks * 32))
    g[:, :cols] = x
    g = g.reshape(rows, blocks, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    top = np.abs(g).max(-1)
    _, e = np.frexp(top)                       # top = f 2^e, f in [0.5, 1)
    e = np.where(top > 0, e - 1 - 2, -127).clip(-127, 127)
    s = np.ldexp(1.0, e)[..., None]
    v = round_to_grid(g / s) * s
    v[bad] = np.nan
    return v.reshape(rows, -1)[:, :cols]


def newton_schulz(G, steps, coefficients, eps):
    a, b, c = coefficients
    G = np.asarray(G, dtype=np.float64)
    out = np.empty_like(G)
    for i in np.ndindex(G.shape[:-2]):
        X = G[i] / (math.sqrt(float((G[i] ** 2).sum())) + eps)
        for _ in range(steps):
            if X.shape[0] <= X.shape[1]:
                S = X @ X.T
                X = a * X + (b * S + c * (S @ S)) @ X
            else:
                S = X.T @ X
                X = a * X + X @ (b * S + c * (S @ S))
        out[i] = X
    return out
