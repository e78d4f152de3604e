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


def to_bfloat16(x):
    """x rounded to the nearest number of bfloat16 (8 significant bits)."""
    f, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(f * 256.0), e - 8)


def held(x, parts):
    """2^12 x as one or two 16-bit floats hold it: the nearest half, and for two
    parts the nearest half of what is left."""
    up = np.asarray(x, dtype=np.float64) * 4096.0
    hi = up.astype(np.float16).astype(np.float64)
    lo = (up - hi).astype(np.float16).astype(np.float64) if parts == 2 else 0.0
    return (hi + lo) / 4096.0


def newton_schulz_held(G, steps, coefficients, eps, parts):
    """newton_schulz of one matrix (rows <= cols) whose iterates, S and b S + c
    S^2 are held in parts; everything between them in 64 bits."""
    a, b, c = coefficients
    G = np.asarray(G, dtype=np.float64)
    X = held(G / (math.sqrt(float((G ** 2).sum())) + eps), parts)
    for i in range(steps):
        S = held(X @ X.T, parts)
        B = held(b * S + c * (S @ S), parts)
        X = a * X + B @ X
        if i + 1 < steps:
            X = held(X, parts)
    return X


def bfloat16_bound(ref, steps):
    """Bound of |got - ref| / |ref| where got is rounded to bfloat16 from numbers
    within d = 12 steps 2^-22 of ref (two parts): a number's distance to the
    type's grid changes by no more than the number does, so rounding costs what
    it costs ref, and d; d itself comes on top."""
    norm = np.linalg.norm(ref)
    return np.linalg.norm(to_bfloat16(ref) - ref) / norm + 2 * 12 * max(steps, 1) * 2.0 ** -22
