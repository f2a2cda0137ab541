"""CPU oracle for the operators whose parameters are matrices (TEST INFRASTRUCTURE ONLY): plain float64 NumPy statements of the
formulas in include/gpga.h.  Parameters come as float32 arrays, activations as whatever values the device holds; nothing is
rounded here.  Pinned by differences and by hand-made cases in tests/test_oracle_matrix_pins.py."""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[float])


def activation(kind, v):
    """(act(v), act'(v))."""
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-v))
        return v * s, s + v * s * (1.0 - s)
    p = 0.5 * (1.0 + _erf(v / math.sqrt(2.0)))
    return v * p, p + v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)


def gated_ff(x, gate, up, down, kind):
    """x (n, T, D), gate and up (n, F, D), down (n, D, F): y, a, b."""
    x, gate, up, down = (np.asarray(v, dtype=np.float64) for v in (x, gate, up, down))
    a, b = x @ gate.transpose(0, 2, 1), x @ up.transpose(0, 2, 1)
    return (activation(kind, a)[0] * b) @ down.transpose(0, 2, 1), a, b


def gated_ff_grad(dy, x, a, b, gate, up, down, kind):
    """dx and the gradients of gate, up and down, from the a and b that were kept."""
    dy, x, a, b, gate, up, down = (np.asarray(v, dtype=np.float64) for v in (dy, x, a, b, gate, up, down))
    value, slope = activation(kind, a)
    dh = dy @ down
    da, db = dh * b * slope, dh * value
    t = lambda v: v.transpose(0, 2, 1)
    return da @ gate + db @ up, t(da) @ x, t(db) @ x, t(dy) @ (value * b)


def orthogonalize(g, v, mu, nesterov, steps, coefficients, eps, scale):
    """g and v (k, rows, cols); v None: no momentum.  (update, new v)."""
    p, q, r = coefficients
    g = np.asarray(g, dtype=np.float64)
    if v is not None:
        v = mu * np.asarray(v, dtype=np.float64) + g
    u = g if v is None else g + mu * v if nesterov else v
    out = []
    for m in u:
        x = m / (np.sqrt((m * m).sum()) + eps)
        x = x if m.shape[0] <= m.shape[1] else x.T
        for _ in range(steps):
            gram = x @ x.T
            x = p * x + (q * gram + r * gram @ gram) @ x
        out.append(scale * (x if m.shape[0] <= m.shape[1] else x.T))
    return np.stack(out), v
