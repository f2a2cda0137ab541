"""Orthogonalised updates on the GPU against the float64 oracle, through the C ABI.

Tolerance.  Everything is held in two fp16 pieces, 2^-22 of a value, products leave out another 2^-22 of a term, sums are fp32: a step
computes p X + (q A + r A^2) X with a perturbation E of the matrix whose entries are independent rounding errors.  With m the shorter
side and singular values up to M, each of the three products is off in 2-norm by at most e = (4 2^-22 + (K + 16) 2^-24 / sqrt K) times
the Frobenius norms of its factors (rounding errors of a sum of K terms: the bound with the square root of K, errors being as often
up as down).  A step's error is amplified by later ones by at most the polynomial's largest slope, P = p where q < 0 < r.  So the 2-norm
of the whole error stays below e (|q| M^2 + |r| M^4 + p) |X| sum of P^k, k < steps, |X| = M sqrt m, and that is asked of the Frobenius norm
of the difference; elements are at most that far off, too.
"""
import numpy as np
import pytest

from oracle import matrix_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


@pytest.fixture(scope="module")
def hx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2105_09080_amd import harness
    return harness


def tolerance(rows, cols, steps, coefficients, scale):
    p, q, r = (abs(v) for v in coefficients)
    m, k, top = min(rows, cols), max(rows, cols), 1.25
    e = 4 * 2.0 ** -22 + (np.sqrt(k) + 16) * 2.0 ** -24
    grown = sum(p ** j for j in range(steps))
    return abs(scale) * e * (q * top ** 2 + r * top ** 4 + p) * top * np.sqrt(m) * grown


def gradients(rng, k, rows, cols, kind):
    g = rng.normal(size=(k, rows, cols))
    if kind == "strong":                                             # a few directions far above the others
        g += 30 * rng.normal(size=(k, rows, 1)) * rng.normal(size=(k, 1, cols))
    if kind == "tiny":
        g *= 1e-33
    if kind == "huge":
        g *= 1e30
    return g.astype(np.float32)


CASES = [  # n, rows, cols, count, off, kind of gradient, momentum, Nesterov, steps, coefficients, scale
    (1, 1, 1, 1, 0, "noise", None, False, 5, QUINTIC, 1.0), (3, 1, 9, 1, 2, "noise", 0.9, False, 5, QUINTIC, 1.0),
    (2, 7, 5, 3, 1, "noise", 0.9, True, 5, QUINTIC, 1.4), (20, 64, 64, 1, 0, "strong", None, False, 5, QUINTIC, 1.0),
    (2, 65, 130, 2, 3, "noise", 0.95, True, 5, QUINTIC, 0.2), (2, 130, 65, 2, 3, "strong", 0.95, False, 5, QUINTIC, 0.2),
    (1, 257, 300, 1, 0, "tiny", None, False, 5, QUINTIC, 1.0), (1, 300, 257, 1, 0, "huge", None, False, 5, QUINTIC, -1.0),
    (3, 40, 600, 1, 7, "noise", 0.5, False, 3, CUBIC, 1.0), (3, 600, 40, 1, 7, "noise", 0.0, False, 8, CUBIC, 1.0),
    (2, 33, 20, 1, 0, "noise", 0.9, True, 0, QUINTIC, 3.0), (2, 128, 128, 2, 0, "noise", None, False, 1, QUINTIC, 1.0),
    (40, 200, 900, 2, 0, "strong", None, False, 5, QUINTIC, 1.0), (40, 520, 300, 2, 1, "noise", 0.95, True, 5, QUINTIC, 1.0),
]


@pytest.mark.parametrize("n,rows,cols,count,off,kind,mu,nesterov,steps,coefficients,scale", CASES)
def test_update(hx, n, rows, cols, count, off, kind, mu, nesterov, steps, coefficients, scale):
    rng = np.random.default_rng(rows + cols + steps)
    size = count * rows * cols
    sim = hx.Simulation(n, off + size + 3, topology="ring", H=4, lr=0.1, ld=off + size + 5)
    before = rng.normal(size=(n, off + size + 3)).astype(np.float32)
    before[:, off:off + size] = gradients(rng, n * count, rows, cols, kind).reshape(n, size)
    v0 = None if mu is None else (0.5 * rng.normal(size=(n, size)) * np.abs(before[:, off:off + size]).max()).astype(np.float32)
    velocity = None if mu is None else torch.as_tensor(v0).cuda()
    sim.set_state(G=before)
    shape = (n * count, rows, cols)
    want, v = orc.orthogonalize(before[:, off:off + size].reshape(shape), None if mu is None else v0.reshape(shape),
                                0.0 if mu is None else float(np.float32(mu)), nesterov, steps, [float(np.float32(c)) for c in coefficients], 1e-7, scale)
    sim.orthogonalize(off, rows, cols, count=count, velocity=velocity, mu=mu or 0.0, nesterov=nesterov, steps=steps,
                      coefficients=coefficients, scale=scale)
    got = sim.G.double().cpu().numpy()
    assert np.array_equal(got[:, :off], before[:, :off]) and np.array_equal(got[:, off + size:], before[:, off + size:])
    far = np.sqrt(((got[:, off:off + size].reshape(shape) - want) ** 2).sum(axis=(1, 2)))
    tol = tolerance(rows, cols, max(steps, 1), coefficients, scale)
    assert far.max() <= tol, (far.max(), tol)
    if mu is not None:
        close = np.abs(velocity.double().cpu().numpy() - v.reshape(n, size)) <= 2.0 ** -23 * (np.abs(mu * v0) + np.abs(before[:, off:off + size]))
        assert close.all()
    sim.close()
