"""Orthogonalised updates whose values grow or shrink far, on the GPU against the float64 oracle: each result by its own size.

Tolerance.  A step's X is held in two fp16 pieces, off by 2^-22 of a value, and made by at most six roundings of fp32: p X off by 2^-20 of its
norm.  (q A + r A^2) X comes from three products, each off by e = 4 2^-22 + (sqrt K + 16) 2^-24 of its factors' norms (roundings as often up as
down).  All these are relative to the value of the step, so k steps of a polynomial in which no singular value grows beside the others
stay within k (2^-20 + 3 e c) of the result's norm, c what the polynomial's other terms are beside p X.
"""
import numpy as np
import pytest

from oracle import matrix_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SHAPES = [(40, 60), (64, 200), (128, 100), (200, 330), (300, 200)]   # by one workgroup, by launches


@pytest.fixture(scope="module")
def hx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2105_09080_amd import harness
    return harness


def run(hx, g, steps, coefficients, eps, scale=1.0, velocity=None, mu=0.0, nesterov=False):
    """(result, oracle's result) of matrices g (n, rows, cols) in float64."""
    n, rows, cols = g.shape
    sim = hx.Simulation(n, rows * cols, topology="ring", H=4, lr=0.1)
    sim.set_state(G=g.reshape(n, -1).astype(np.float32))
    v = None if velocity is None else torch.as_tensor(velocity.reshape(n, -1).astype(np.float32)).cuda()
    sim.orthogonalize(0, rows, cols, steps=steps, coefficients=coefficients, eps=eps, scale=scale, velocity=v, mu=mu, nesterov=nesterov)
    got = sim.G.double().cpu().numpy().reshape(g.shape)
    sim.close()
    f32 = lambda c: float(np.float32(c))
    want, _ = orc.orthogonalize(g.astype(np.float32), None if velocity is None else velocity.astype(np.float32), f32(mu), nesterov, steps,
                                [f32(c) for c in coefficients], f32(eps), f32(scale))
    return got, want


def norm(v):
    return np.sqrt((v * v).sum(axis=(1, 2)))


def sums(k):
    return 4 * 2.0 ** -22 + (np.sqrt(k) + 16) * 2.0 ** -24


@pytest.mark.parametrize("steps,coefficients,c,scale", [(30, (0.1, 0.0, 0.0), 0.0, 1.0), (9, (0.01, 0.0, 0.0), 0.0, 1.0), (64, (0.5, 0.0, 0.0), 0.0, 1.0),
                                                        (40, (0.5, -0.1, 0.05), 0.3, 1.0), (20, (0.3, 0.2, 0.0), 0.7, -1e5), (64, (0.1, 0.0, 0.0), 0.0, 1e30),
                                                        (5, (2.0, 0.0, 0.0), 0.0, 1e-30), (3, (0.0, 0.0, 0.0), 0.0, 1.0), (64, (0.01, 0.01, 0.01), 2.0, 1.0)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_values_that_shrink_and_grow(hx, rows, cols, steps, coefficients, c, scale):
    g = np.random.default_rng(rows + steps).normal(size=(2, rows, cols))
    got, want = run(hx, g, steps, coefficients, 0.0, scale)
    tol = steps * (2.0 ** -20 + 3 * sums(max(rows, cols)) * c) * norm(want) + 2.0 ** -149 * np.sqrt(rows * cols)
    assert np.isfinite(got).all()
    assert (norm(got - want) <= tol).all(), (norm(got - want) / np.maximum(norm(want), 1e-300)).max()


@pytest.mark.parametrize("n,rows,cols", [(4, 40, 60), (4, 60, 250), (4, 120, 100), (4, 64, 400), (4, 130, 200), (4, 330, 200), (40, 520, 300), (16, 1024, 1024), (8, 700, 2048)])
@pytest.mark.parametrize("p,steps", [(0.77, 3), (0.01, 9), (1.3, 4)])
def test_both_pieces_of_every_element(hx, n, rows, cols, p, steps):
    """X <- p X: every element by itself, 2^-20 of it a step, and what falls below the subnormals of the largest, 2^-36 of the norm.  A second
    piece that does not go with the first leaves 2^-11."""
    g = np.random.default_rng(rows).normal(size=(n, rows, cols)).astype(np.float32)
    sim = hx.Simulation(n, rows * cols, topology="ring", H=4, lr=0.1)
    sim.set_state(G=g.reshape(n, -1))
    sim.orthogonalize(0, rows, cols, steps=steps, coefficients=(p, 0.0, 0.0), eps=0.0, scale=0.9)
    got = sim.G.double().cpu().numpy().reshape(g.shape)
    sim.close()
    g = g.astype(np.float64)
    want = g / norm(g)[:, None, None] * float(np.float32(p)) ** steps * float(np.float32(0.9))
    off = np.abs(got - want) / ((steps + 2) * (2.0 ** -20 * np.abs(want) + 2.0 ** -36 * norm(want)[:, None, None]))
    bad = int((off > 1).sum())
    assert bad == 0, (bad, float(off.max()))


@pytest.mark.parametrize("factor", [1e3, 1e5, 1e9, 1e20])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_eps_far_above_the_norm(hx, rows, cols, factor):
    """X0 = U / (|U| + eps) is small then: five steps make it p^5 as large and little else (c: 4.775 / 3.4445 of the square of a
    singular value, at most 1e-3 * 3.4445^5 / 5 or so).  In the same call matrices far above eps."""
    rng = np.random.default_rng(rows)
    coefficients = (3.4445, -4.7750, 2.0315)
    g = rng.normal(size=(4, rows, cols))
    g /= norm(g)[:, None, None]
    g[1] *= 1e4 * factor
    g[2] = 0.0
    got, want = run(hx, g, 5, coefficients, factor)
    assert not got[2].any()
    tol = 5 * (2.0 ** -20 + 3 * sums(max(rows, cols)) * 0.1) * norm(want)
    off = norm(got - want)
    for i in (0, 3):
        assert off[i] <= tol[i], off[i] / norm(want)[i]
    assert np.isfinite(got).all() and off[1] <= 1e-4 * norm(want)[1]
    velocity = rng.normal(size=g.shape) * 1e-2
    got, want = run(hx, g, 5, coefficients, factor, velocity=velocity, mu=0.9, nesterov=True)
    off = norm(got - want)
    assert (off[[0, 2, 3]] <= (tol[0] / norm(want)[0] + 2.0 ** -22) * 2 * norm(want)[[0, 2, 3]]).all(), off / norm(want)
