"""Performance cases of the matrix operators for training and serving in 4 bits.

Four operators next to the tensor contraction, as their users call them:

- `quantize`: a matrix becomes microscaled 4-bit numbers (E2M1 codes, one E8M0
  scale for 32 neighbours along the axis that a product sums over), along its
  rows, its columns, or both at once, and is read back as values;
- `product`: C = A B^T of two packed matrices;
- `linear`: a packed weight applied to activations in 16 or 32 bits, which are
  quantised in the call (serving), and a training step of a linear layer with
  its three products in 4 bits (y, dx and dw);
- `orthogonalize`: an update matrix becomes nearly orthogonal by five
  Newton-Schulz steps X <- a X + (b X X^T + c (X X^T)^2) X.

Where `own` is false, `run` computes the operators in plain torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ITEM = {"f32": 4, "bf16": 2, "f16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
STEPS = 5


# ------------------------------------------------------------------ cases ---

def _quantize(name, dtype, rows, cols, axis, order="row"):
    return _named(name, {"op": "quantize", "dtype": dtype, "rows": rows, "cols": cols,
                         "axis": axis, "order": order})


def _product(name, dtype, m, n, k):
    return _named(name, {"op": "product", "dtype": dtype, "m": m, "n": n, "k": k})


def _linear(name, dtype, m, n, k, train):
    return _named(name, {"op": "linear", "dtype": dtype, "m": m, "n": n, "k": k, "train": train})


def _orth(name, dtype, batch, rows, cols):
    return _named(name, {"op": "orthogonalize", "dtype": dtype, "batch": batch, "rows": rows,
                         "cols": cols})


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # the activations of a single token: the smallest call, all latency
        _quantize("quantize_token_bf16", "bf16", 1, 4096, "cols"),
        # a weight slice of odd extents inside a wider matrix, packed in both
        # orientations for the products of a training step
        _quantize("quantize_odd_f32", "f32", 1001, 1187, "both", "slice"),
        # the activations of a large training batch, both orientations
        _quantize("quantize_large_bf16", "bf16", 16384, 8192, "both"),
        # sixteen sequences decoded together: bound by the weight's bytes
        _product("product_few_bf16", "bf16", 16, 8192, 4096),
        # a ragged product: no extent fits a tile, K ends inside a block
        _product("product_odd_f32", "f32", 777, 1250, 1999),
        # the product of a long prompt or a training batch
        _product("product_large_bf16", "bf16", 8192, 8192, 8192),
        # a linear layer for one token
        _linear("linear_token_bf16", "bf16", 1, 8192, 4096, False),
        # a training step of a layer of odd widths in 32 bits
        _linear("linear_step_odd_f32", "f32", 1023, 515, 1000, True),
        # a training step of a wide layer
        _linear("linear_step_bf16", "bf16", 8192, 8192, 4096, True),
        # the heads' slices of a small weight, one matrix each
        _orth("orth_heads_f32", "f32", 12, 64, 128),
        # a tall matrix of odd extents
        _orth("orth_odd_bf16", "bf16", 1, 1000, 517),
        # the square weight of a wide layer
        _orth("orth_large_f32", "f32", 1, 4096, 4096),
    ]


def _size(rng, low, high):
    """log-uniform in [low, high]; half of the larger ones multiples of 32"""
    v = round(math.exp(rng.uniform(math.log(low), math.log(high))))
    if v >= 64 and rng.random() < 0.5:
        v = 32 * round(v / 32)
    return max(low, min(high, v))


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "f16"))
    op = rng.choice(("quantize", "product", "linear", "step", "orthogonalize"))
    if op == "quantize":
        return _quantize(None, dtype, _size(rng, 1, 16384), _size(rng, 1, 8192),
                         rng.choice(("rows", "cols", "both")), rng.choice(("row", "col", "slice")))
    if op == "product":
        return _product(None, dtype, _size(rng, 1, 8192), _size(rng, 16, 8192),
                        _size(rng, 16, 8192))
    if op == "linear":
        return _linear(None, dtype, _size(rng, 1, 8192), _size(rng, 16, 8192),
                       _size(rng, 16, 4096), False)
    if op == "step":
        return _linear(None, dtype, _size(rng, 1, 8192), _size(rng, 16, 8192),
                       _size(rng, 16, 4096), True)
    rows, cols = _size(rng, 16, 4096), _size(rng, 16, 4096)
    batch = _size(rng, 1, 16) if rows * cols <= 1 << 18 else 1
    return _orth(None, dtype, batch, rows, cols)


# ----------------------------------------------------------------- inputs ---

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _activations(gen, rows, cols, dtype):
    """Normal values, every channel with a size of its own (e^N(0,1)): the
    blocks' scales differ as those of activations do."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp(torch.randn(1, cols, generator=gen, device="cuda"))
    return x.to(TORCH[dtype])


def _weights(gen, rows, cols, dtype):
    return (torch.randn(rows, cols, generator=gen, device="cuda") / math.sqrt(cols)).to(TORCH[dtype])


def _inputs(case, seed):
    gen, dt = _generator(seed), case["dtype"]
    if case["op"] == "quantize":
        r, c = case["rows"], case["cols"]
        if case["order"] == "col":
            return (_activations(gen, c, r, dt).t(),)
        if case["order"] == "slice":
            return (_activations(gen, r, c + 13, dt)[:, 5:5 + c],)
        return (_activations(gen, r, c, dt),)
    if case["op"] == "orthogonalize":
        # a momentum buffer: a few strong directions over noise
        b, r, c = case["batch"], case["rows"], case["cols"]
        rank = max(1, min(r, c) // 16)
        u = torch.randn(b, r, rank, generator=gen, device="cuda")
        v = torch.randn(b, rank, c, generator=gen, device="cuda")
        g = (u @ v) / math.sqrt(rank) + torch.randn(b, r, c, generator=gen, device="cuda")
        return ((1e-3 * g).to(TORCH[dt]),)
    m, n, k = case["m"], case["n"], case["k"]
    x, w = _activations(gen, m, k, dt), _weights(gen, n, k, dt)
    if case["op"] == "linear" and case["train"]:
        return x, w, _activations(gen, m, n, dt) * 1e-3
    return x, w


def prepare(case, seed):
    """What the program keeps: float matrices, and for the products the packed
    operands (for serving only the weight)."""
    state = {"case": case, "own": own}
    t = _inputs(case, seed)
    packed = _packed_operands(case)
    if own:
        import paper_1607_00145_amd as gett
        state["gett"] = gett
        pack = gett.mx_quantize
    else:
        pack = _plain_pack
    state["in"] = [pack(x) if i in packed else x for i, x in enumerate(t)]
    return state


def _packed_operands(case):
    if case["op"] == "product":
        return (0, 1)
    return (1,) if case["op"] == "linear" and not case["train"] else ()


# ------------------------------------------------------------- plain forms ---

_POW2 = {}


def _pow2(e, device):
    """2^e for integers in [-127, 127]"""
    if device not in _POW2:
        _POW2[device] = torch.tensor([2.0 ** k for k in range(-127, 128)], dtype=torch.float32,
                                     device=device)
    return _POW2[device][e + 127]


def _plain_codes(x):
    """[rows, K] -> magnitudes' codes 0..7 with the sign as bit 3, [rows, blocks,
    32], and the blocks' exponents"""
    x = x.float()
    pad = -x.shape[1] % 32
    if pad:
        x = torch.cat((x, x.new_zeros(x.shape[0], pad)), 1)
    x = x.reshape(x.shape[0], -1, 32)
    a = x.abs()
    top = a.amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(-127, 127)      # floor(log2 top) - 2
    a = a * _pow2(-e, x.device)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0))
    return code + 8 * (x < 0).to(torch.uint8), e.squeeze(-1)


def _plain_pack(x):
    code, e = _plain_codes(x)
    code = code.reshape(code.shape[0], -1)
    return {"codes": code[:, 0::2] | (code[:, 1::2] << 4), "exponents": e, "k": x.shape[1]}


def _plain_values(codes, e, k):
    """codes [rows, blocks, 32] -> float32 [rows, k]"""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float32,
                         device=codes.device)
    table = torch.cat((table, -table))
    v = table[codes.int()] * _pow2(e, codes.device)[..., None]
    return v.reshape(v.shape[0], -1)[:, :k]


def _plain_unpack(p):
    c = torch.stack((p["codes"] & 15, p["codes"] >> 4), -1)
    return _plain_values(c.reshape(c.shape[0], -1, 32), p["exponents"], p["k"])


def _plain_round(x):
    return _plain_values(*_plain_codes(x), x.shape[1])


def _value_type(case):
    # 4-bit values with their scale are numbers of bfloat16 (not of float16)
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _run_plain(case, t):
    dt = TORCH[case["dtype"]]
    if case["op"] == "quantize":
        x, vt = t[0], _value_type(case)
        out = []
        if case["axis"] in ("cols", "both"):
            out.append(_plain_round(x).to(vt))
        if case["axis"] in ("rows", "both"):
            out.append(_plain_round(x.t()).to(vt))
        return out
    if case["op"] == "product":
        return _plain_unpack(t[0]).matmul(_plain_unpack(t[1]).t()).to(dt)
    if case["op"] == "linear" and not case["train"]:
        return _plain_round(t[0]).matmul(_plain_unpack(t[1]).t()).to(dt)
    if case["op"] == "linear":
        x, w, dy = t
        y = _plain_round(x).matmul(_plain_round(w).t())
        dx = _plain_round(dy).matmul(_plain_round(w.t()).t())
        dw = _plain_round(dy.t()).matmul(_plain_round(x.t()).t())
        return y.to(dt), dx.to(dt), dw.to(dt)
    a, b, c = COEFFICIENTS
    X = t[0].float()
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2).contiguous()
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        A = X.matmul(X.transpose(1, 2))
        X = a * X + (b * A + c * A.matmul(A)).matmul(X)
    return (X.transpose(1, 2) if tall else X).to(dt)


# -------------------------------------------------------------------- runs ---

def _run_own(gett, case, t):
    dt = TORCH[case["dtype"]]
    if case["op"] == "quantize":
        q = gett.mx_quantize(t[0], along=case["axis"])
        return [p.dequantize(_value_type(case)) for p in (q if case["axis"] == "both" else (q,))]
    if case["op"] == "product" or not case.get("train", True):
        return gett.mx_matmul(t[0], t[1], dtype=dt)
    if case["op"] == "linear":
        x, w, dy = t
        x = x.detach().requires_grad_()
        w = w.detach().requires_grad_()
        y = gett.mx_linear(x, w)
        dx, dw = torch.autograd.grad(y, (x, w), dy)
        return y.detach(), dx, dw
    return gett.orthogonalize(t[0], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)


def run(state):
    if state["own"]:
        return _run_own(state["gett"], state["case"], state["in"])
    return _run_plain(state["case"], state["in"])


# -------------------------------------------------------------------- work ---

def _packed_bytes(rows, k):
    blocks = -(-k // 32)
    return rows * blocks * 17


def work(case):
    item = ITEM[case["dtype"]]
    if case["op"] == "quantize":
        r, c = case["rows"], case["cols"]
        n = item * r * c
        out = 2 if case["dtype"] == "bf16" else 4
        for axis, size in (("cols", (r, c)), ("rows", (c, r))):
            if case["axis"] in (axis, "both"):      # packed, read back, values written
                n += 2 * _packed_bytes(*size) + out * r * c
        return {"bytes": n, "flops": 0}
    if case["op"] == "orthogonalize":
        b, r, c = case["batch"], case["rows"], case["cols"]
        m, n = min(r, c), max(r, c)
        # X X^T and its square are symmetric: half of each
        per = m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n
        return {"bytes": 2 * item * b * r * c, "flops": STEPS * b * per}
    m, n, k = case["m"], case["n"], case["k"]
    flops = 2 * m * n * k
    if case["op"] == "product":
        return {"bytes": _packed_bytes(m, k) + _packed_bytes(n, k) + item * m * n, "flops": flops}
    if not case["train"]:
        return {"bytes": item * m * k + _packed_bytes(n, k) + item * m * n, "flops": flops}
    # x, w, dy read; y, dx, dw written; the layer keeps no packed copies
    return {"bytes": 2 * item * (m * k + n * k + m * n), "flops": 3 * flops}


# ------------------------------------------------------------------- exact ---

def _exact_round(x):
    """Microscaled values of [rows, K] in 64 bits: the multiple of the local
    step that is nearest, ties to the even multiple, at most 6 scales."""
    x = x.double()
    rows, k = x.shape
    out = torch.zeros(rows, -(-k // 32) * 32, dtype=torch.float64, device=x.device)
    out[:, :k] = x
    g = out.view(rows, -1, 32)
    top = g.abs().max(2, keepdim=True).values
    shift = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2
    scale = torch.exp2(shift.clamp(-127, 127))
    q = g / scale
    size = q.abs()
    binade = torch.floor(torch.log2(torch.where(size > 1, size, torch.ones_like(size))))
    step = torch.exp2(binade - 1)
    q = (torch.round(q / step) * step).clamp(-6, 6)
    return (q * scale).reshape(rows, -1)[:, :k].contiguous()


def exact(case, seed):
    t = _inputs(case, seed)
    if case["op"] == "quantize":
        ways = {"cols": (t[0],), "rows": (t[0].t(),), "both": (t[0], t[0].t())}
        return [_exact_round(x) for x in ways[case["axis"]]]
    if case["op"] == "orthogonalize":
        a, b, c = COEFFICIENTS
        out = torch.empty(t[0].shape, dtype=torch.float64, device="cuda")
        for i, G in enumerate(t[0].double()):
            wide = G if G.shape[0] <= G.shape[1] else G.t().contiguous()
            Y = wide / (torch.linalg.vector_norm(wide) + EPS)
            eye = torch.eye(Y.shape[0], dtype=torch.float64, device="cuda")
            for _ in range(STEPS):
                P = torch.mm(Y, Y.t().contiguous())
                Y = torch.mm(a * eye + torch.mm(P, b * eye + c * P), Y)
            out[i] = Y if G.shape[0] <= G.shape[1] else Y.t()
        return out
    x, w = t[0], t[1]
    y = torch.mm(_exact_round(x), _exact_round(w).t().contiguous())
    if case["op"] == "product" or not case["train"]:
        return y
    dy = t[2]
    dx = torch.mm(_exact_round(dy), _exact_round(w.t()).t().contiguous())
    dw = torch.mm(_exact_round(dy.t()), _exact_round(x.t()).t().contiguous())
    return y, dx, dw
