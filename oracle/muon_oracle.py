"""CPU oracle for orthogonalised updates.  TEST INFRASTRUCTURE ONLY.

Only tests/, __graft_entry__.smoke() and the cpu_baseline leg of bench.py may import this module.  It shares no code with the
HIP library and never imports it.  Float64 numpy.

Newton-Schulz: X = G / (|G|_F + eps), then X <- a X + b (X X^T) X + c (X X^T)^2 X with the coefficients that the Muon optimiser
published.  A step maps every singular value s of X to a s + b s^3 + c s^5 and leaves the singular vectors, so the result also has
a closed form by the singular value decomposition, which the pins compare (tests/test_oracle_muon_pins.py).

Muon step: m <- mu m + (1 - mu) g;  u = (1 - mu) g + mu m (Nesterov) or m;  p <- (1 - lr wd) p - lr rms sqrt(max(rows, cols)) O(u).
"""
from __future__ import annotations

import math

import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def newton_schulz(g, steps=5, eps=1e-7):
    x = np.asarray(g, np.float64)
    x = x / (math.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            s = x @ x.T
            x = A * x + B * (s @ x) + C * (s @ (s @ x))
        else:
            s = x.T @ x
            x = A * x + B * (x @ s) + C * ((x @ s) @ s)
    return x


def muon_step(p, g, m, lr, momentum=0.95, nesterov=True, weight_decay=0.01, rms=0.2, steps=5, eps=1e-7, grad_scale=1.0):
    """Returns (p, m, O) after the step, float64."""
    p, m = np.asarray(p, np.float64), np.asarray(m, np.float64)
    g = np.asarray(g, np.float64) * grad_scale
    m = momentum * m + (1.0 - momentum) * g
    o = newton_schulz((1.0 - momentum) * g + momentum * m if nesterov else m, steps, eps)
    return p * (1.0 - lr * weight_decay) - lr * rms * math.sqrt(max(p.shape)) * o, m, o
