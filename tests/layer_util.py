"""Plain 64-bit forms of the operators of a feed-forward layer, for their tests:
written from the definitions in include/gett_layers.h, on the CPU, sharing nothing
with the library; and bounds of what its arithmetic may be off by.

Bounds are element by element.  u is half a step of the type (2^-8, 2^-11, 2^-24
relative), v = 2^-24 that of the sums.  A sum of K products in 32 bits is off by at
most (K + 2) v sum|x w| (each product and each addition rounds once, in any order).
"""
from __future__ import annotations

import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
V = 2.0 ** -24
# numbers below this are multiples of the type's least step, which bounds their rounding
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def philox(c, key):
    """Philox4x32-10 of counters [..., 4] (numpy, whole numbers)."""
    c = [c[..., i].astype(object) for i in range(4)]
    k0, k1 = key & 0xffffffff, key >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k0, b & 0xffffffff, (a >> 32) ^ c[3] ^ k1, a & 0xffffffff]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return np.stack(c, -1)


def mask(rows, cols, p, seed, offset):
    """The factors of a rows x cols matrix: 0 or 1 / (1 - p), p a multiple of 2^-16."""
    cut = round(p * 65536)
    if cut == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    groups = -(-cols // 8)
    c = np.zeros((rows, groups, 4), dtype=object)
    c[..., 0] = np.arange(groups)[None]
    c[..., 1] = np.arange(rows)[:, None]
    c[..., 2], c[..., 3] = offset & 0xffffffff, offset >> 32 & 0xffffffff
    words = philox(c, seed & (1 << 64) - 1).astype(np.int64)
    fields = np.stack((words & 0xffff, words >> 16), -1).reshape(rows, groups * 8)[:, :cols]
    scale = 65536.0 / (65536 - cut) if cut < 65536 else 0.0
    return torch.from_numpy((fields >= cut) * scale)


def act(name, z):
    """act(z), its slope and a bound of the slope's own slope, in 64 bits."""
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), 0.0
    if name == "gelu":
        cdf, pdf = torch.special.ndtr(z), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return z * cdf, cdf + z * pdf, 0.8      # (2 - z^2) pdf
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s)), 0.5
    return z, torch.ones_like(z), 0.0


# an activation's value and slope in 32 bits: a few operations on numbers of their
# size, exp and erf of two steps each
def act_error(z):
    return 16 * V * (1 + z.abs())


def linear(x, w, bias, name, keep, residual, dtype):
    """y and a bound of its error, z and a bound of its error, in 64 bits."""
    x, w = x.double(), w.double()
    k = x.shape[1]
    z = x @ w.t()
    size = x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    dz = (k + 4) * V * size
    a, s, s2 = act(name, z)
    # slopes are at most 1.13; what is beyond the first order is below 1e-6 of it
    da = 1.14 * dz + (act_error(z) * (z.abs() if name else 0) if name else 0)
    y = a * keep
    r = 0.0 if residual is None else residual.double()
    dy = da * keep + 4 * V * (y.abs() + (r.abs() if residual is not None else 0))
    y = y + r
    return y, dy + rounding(y.abs() + dy, dtype), z, dz


def rounding(x, dtype):
    return U[dtype] * x + TINY[dtype]


def linear_grads(dy, x, w, z, dz_error, name, keep, dtype):
    """dx, dw, dbias and bounds of their errors.  dz is taken at the rounded z and
    rounded itself; dbias before that."""
    dy, x, w = dy.double(), x.double(), w.double()
    _, s, s2 = act(name, z)
    g = dy * keep
    dz = g * s
    off_z = dz_error + (rounding(z.abs() + dz_error, dtype) if name else 0)
    err = g.abs() * (s2 * off_z + (act_error(z) if name else 0)) + 4 * V * dz.abs()
    m, n = dy.shape
    db, db_err = dz.sum(0), err.sum(0) + (m + 2) * V * dz.abs().sum(0)
    err = err + rounding(dz.abs() + err, dtype)
    dx, dw = dz @ w, dz.t() @ x
    big = dz.abs() + err
    dx_err = err @ w.abs() + (n + 2) * V * (big @ w.abs())
    dw_err = err.t() @ x.abs() + (m + 2) * V * (big.t() @ x.abs())
    return [(v, e + rounding(v.abs() + e, dtype)) for v, e in
            ((dx, dx_err), (dw, dw_err), (db, db_err))]


def close(got, ref, err, what=""):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~((got - ref).abs() <= err)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(),
                           float(((got - ref).abs() / err)[bad].max()))


# routing ---------------------------------------------------------------------

def route(logits, k, scoring, bias=None, groups=1, top_groups=None, renormalize=True, scale=1.0):
    """weights (64 bits), index, order, offsets, place; token by token."""
    x = logits.detach().double().cpu().numpy()
    t, e = x.shape
    top_groups = groups if top_groups is None else top_groups
    weights, index = np.zeros((t, k)), np.full((t, k), -1)
    for i in range(t):
        v = np.where(np.isnan(x[i]), -np.inf, x[i])
        with np.errstate(all="ignore"):
            if scoring == "softmax":
                s = np.where(v == -np.inf, 0.0, np.exp(v - v.max()))
                s = s / s.sum()
            else:
                s = 1 / (1 + np.exp(-v))
            key = v if bias is None and groups == 1 else s + (0 if bias is None else
                                                             bias.double().cpu().numpy())
        key = np.where((v == -np.inf) | np.isnan(key), -np.inf, key)
        if groups > 1:
            parts = key.reshape(groups, -1)
            top = -np.sort(-parts, 1)[:, :2]
            best = np.where(top == -np.inf, 0, top).sum(1)
            best = np.where(top[:, 0] == -np.inf, -np.inf, best)
            kept = np.argsort(-best, kind="stable")[:top_groups]
            closed = np.ones(groups, bool)
            closed[kept] = False
            key = np.where(np.repeat(closed, e // groups), -np.inf, key)
        pick = np.argsort(-key, kind="stable")[:k]
        pick = pick[key[pick] > -np.inf]
        index[i, :len(pick)] = pick
        w = s[pick]
        if renormalize and len(pick) and scoring == "softmax" and v.max() < np.inf:
            w = np.exp(v[pick] - v[pick].max())   # (the same ratios, which do not vanish)
        if renormalize and len(pick):
            w = w / w.sum() if w.sum() > 0 or np.isnan(w.sum()) else np.zeros_like(w)
        weights[i, :len(pick)] = w * scale
        if np.isnan(x[i]).any() or (scoring == "softmax" and (x[i] == np.inf).any()):
            weights[i] = np.nan
    flat = index.reshape(-1)
    order = np.concatenate([np.nonzero(flat == j)[0] for j in range(e)] or [np.zeros(0, int)])
    offsets = np.concatenate(([0], np.cumsum([(flat == j).sum() for j in range(e)])))
    place = np.full(t * k, -1)
    place[order] = np.arange(len(order))
    order = np.concatenate((order, np.full(t * k - len(order), -1)))
    return weights, index, order, offsets, place.reshape(t, k)
