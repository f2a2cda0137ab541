"""Orthogonalised updates to within what two pieces of every operand make possible: a tolerance that a result made of one piece, or of products
without the second pieces, does not meet (shown here on the CPU), over the cases of the broader test.

Tolerance.  The X of every step is off by at most E = 2^-21 + sqrt(K) 2^-25 of its norm: two pieces (2^-22), what products leave out (2^-22), fp32 sums of
K terms.  An error in X_j grows by at most G a step, the largest of (f(s) - f(t)) / (s - t) and (f(s) + f(t)) / (s + t) over the
singular values s, t and 0 (the polynomial's derivative as a function of a matrix), f(s) = p s + q s^3 + r s^5.  So the result is off by at most
E (|X_0| G_0 G_1 .. + |X_1| G_1 .. + .. + |X_last|) in the Frobenius norm.
"""
import numpy as np
import pytest

from oracle import matrix_oracle as orc
from test_gpu_orthogonalize import CASES, gradients

MATRICES = 4  # of a case's that are looked at


def f32(v):
    return float(np.float32(v))


def growth(s, p, q, r):
    s = np.append(s, 0.0)
    f = p * s + q * s ** 3 + r * s ** 5
    a, b = s[:, None], s[None, :]
    total = a + b
    plus = np.where(total > 0, (f[:, None] + f[None, :]) / np.where(total > 0, total, 1.0), p)
    minus = p + q * (a * a + a * b + b * b) + r * (a ** 4 + a ** 3 * b + a * a * b * b + a * b ** 3 + b ** 4)
    return max(np.abs(plus).max(), np.abs(minus).max()), f[:-1]


def tolerance(x0, steps, coefficients):
    s = np.linalg.svd(x0, compute_uv=False)
    E = 2.0 ** -21 + np.sqrt(max(x0.shape)) * 2.0 ** -25
    off = E * np.linalg.norm(s)
    for _ in range(steps):
        G, s = growth(s, *coefficients)
        off = off * G + E * np.linalg.norm(s)
    return off


def case(index):
    n, rows, cols, count, off, kind, mu, nesterov, steps, coefficients, scale = CASES[index]
    rng = np.random.default_rng(rows + cols + steps)
    size = count * rows * cols
    before = rng.normal(size=(n, off + size)).astype(np.float32)
    before[:, off:] = gradients(rng, n * count, rows, cols, kind).reshape(n, size)
    v0 = None if mu is None else (0.5 * rng.normal(size=(n, size)) * np.abs(before[:, off:]).max()).astype(np.float32)
    eps = 0.0 if kind == "tiny" else 1e-7
    return before, v0, eps


def starts(before, v0, index, eps):
    """X_0 of the matrices that are looked at, without the oracle's steps."""
    n, rows, cols, count, off, kind, mu, nesterov, steps, coefficients, scale = CASES[index]
    shape = (n * count, rows, cols)
    pick = np.unique(np.linspace(0, n * count - 1, MATRICES).astype(int))
    g = before[:, off:].reshape(shape)[pick]
    v = None if v0 is None else v0.reshape(shape)[pick]
    return pick, g, v, orc.orthogonalize(g, v, 0.0 if mu is None else f32(mu), nesterov, 0, (1.0, 0.0, 0.0), f32(eps), 1.0)[0]


def one_piece(x, steps, coefficients):
    half = lambda v: v.astype(np.float16).astype(np.float64)
    p, q, r = coefficients
    x = x if x.shape[0] <= x.shape[1] else x.T
    for _ in range(steps):
        h = half(x * 2.0 ** 13) / 2.0 ** 13
        a = h @ h.T
        a1 = half(a * 2.0 ** 13) / 2.0 ** 13
        b = half((q * a + r * a1 @ a1) * 2.0 ** 12) / 2.0 ** 12
        x = p * h + b @ h
    return x


STEPS = [i for i, c in enumerate(CASES) if c[8] > 0]


@pytest.mark.parametrize("index", STEPS)
def test_one_piece_would_not_do(index):
    n, rows, cols, count, off, kind, mu, nesterov, steps, coefficients, scale = CASES[index]
    coefficients = [f32(c) for c in coefficients]
    before, v0, eps = case(index)
    _, _, _, x0 = starts(before, v0, index, eps)
    for x in x0:
        tol = tolerance(x, steps, coefficients)
        want = orc.orthogonalize(x[None], None, 0.0, False, steps, coefficients, 0.0, 1.0)[0][0]
        got = one_piece(x / np.linalg.norm(x), steps, coefficients)
        got = got if rows <= cols else got.T
        assert tol < 1e-3 * max(1.0, np.linalg.norm(want))           # a result of zeros fails, too
        if min(rows, cols) > 1:                                      # one number has one rounding, which may be none
            assert np.linalg.norm(got - want) > 2 * tol, (np.linalg.norm(got - want), tol)


@pytest.mark.gpu
@pytest.mark.parametrize("index", range(len(CASES)))
def test_update_has_both_pieces(index):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2105_09080_amd import harness
    n, rows, cols, count, off, kind, mu, nesterov, steps, coefficients, scale = CASES[index]
    before, v0, eps = case(index)
    size = count * rows * cols
    sim = harness.Simulation(n, off + size, topology="ring", H=4, lr=0.1)
    sim.set_state(G=before)
    velocity = None if v0 is None else torch.as_tensor(v0).cuda()
    sim.orthogonalize(off, rows, cols, count=count, velocity=velocity, mu=mu or 0.0, nesterov=nesterov, steps=steps, coefficients=coefficients, eps=eps,
                      scale=scale)
    got = sim.G.double().cpu().numpy()[:, off:].reshape(n * count, rows, cols)
    sim.close()
    coefficients = [f32(c) for c in coefficients]
    pick, g, v, x0 = starts(before, v0, index, eps)
    want, _ = orc.orthogonalize(g, v, 0.0 if mu is None else f32(mu), nesterov, steps, coefficients, f32(eps), f32(scale))
    for k, i in enumerate(pick):
        far, tol = np.linalg.norm(got[i] - want[k]), abs(scale) * tolerance(x0[k], steps, coefficients)
        assert far <= tol, (int(i), far, tol)
