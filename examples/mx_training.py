"""Train a small network whose products run in 4 bits, then serve it in 4 bits.

    python examples/mx_training.py [--steps N]

A two-layer regression network learns a random teacher's outputs.  Every
product of the forward and the backward pass is `mx_linear`; the update of a
weight is its momentum, made orthogonal by `orthogonalize`.  Afterwards the
weights are packed once with `mx_quantize` and single rows go through
`mx_linear` with the packed weights, quantised on their way in.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1607_00145_amd as gett  # noqa: E402


def forward(x, weights):
    """Hidden layers with a ReLU, a linear last one; float or packed weights."""
    for w in weights[:-1]:
        x = gett.mx_linear(x, w).relu()
    return gett.mx_linear(x, weights[-1])


def train(steps=60, width=256, batch=512, rate=0.05, momentum=0.9, seed=0, log=None):
    """Returns the trained weights, the inputs and the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    teacher = [randn(width, 96) / 96 ** 0.5, randn(32, width) / width ** 0.5]
    x = randn(batch, 96)
    target = torch.relu(x @ teacher[0].t()) @ teacher[1].t()
    weights = [(0.5 * randn(*t.shape) / t.shape[1] ** 0.5).requires_grad_() for t in teacher]
    moments = [torch.zeros_like(w) for w in weights]
    losses = []
    for step in range(steps):
        loss = (forward(x, weights) - target).square().mean()
        grads = torch.autograd.grad(loss, weights)
        with torch.no_grad():
            for w, m, g in zip(weights, moments, grads):
                m.mul_(momentum).add_(g)
                update = gett.orthogonalize(m)
                # an orthogonal matrix of n rows moves outputs by about 1
                scale = rate * max(1.0, w.shape[0] / w.shape[1]) ** 0.5 * (1.0 - step / steps)
                w.sub_(update, alpha=scale)
        losses.append(float(loss.detach()))
        if log and step % 10 == 0:
            log(f"step {step:3d}  loss {losses[-1]:.4f}")
    return [w.detach() for w in weights], x, losses


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    weights, x, losses = train(steps=a.steps, log=print)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    packed = [gett.mx_quantize(w) for w in weights]
    kept = sum(q.codes.numel() + q.scales.numel() for q in packed)
    print(f"weights: {sum(w.numel() * 4 for w in weights)} bytes, packed {kept}")
    one, many = forward(x[:1], packed), forward(x, weights)[:1]
    print(f"one row served in 4 bits, against the batch: {float((one - many).abs().max()):.2e}")


if __name__ == "__main__":
    main()
