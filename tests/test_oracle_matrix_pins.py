"""Pins of the oracle for the operators whose parameters are matrices: gradients against differences, hand-made cases."""
import numpy as np
import pytest

from oracle import matrix_oracle as orc


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activation_and_its_slope(kind):
    v = np.array([-9.0, -1.0, -1e-3, 0.0, 0.5, 3.0, 20.0])
    value, slope = orc.activation(kind, v)
    e = 1e-6
    assert np.allclose(slope, (orc.activation(kind, v + e)[0] - orc.activation(kind, v - e)[0]) / (2 * e), atol=1e-8)
    assert value[3] == 0.0 and slope[3] == 0.5 and abs(value[6] - 20.0) < 1e-6
    known = {"silu": 1 / (1 + np.exp(-1)) - 1, "gelu": -0.15865525393145707}     # act(-1): -sigmoid(-1), -Phi(-1)
    assert abs(value[1] - known[kind]) < 1e-15


def test_forward_by_hand():
    one = lambda *v: np.array(v, dtype=float)
    y, a, b = orc.gated_ff(one(2.0, 3.0).reshape(1, 1, 2), one(1, 0).reshape(1, 1, 2), one(0, 1).reshape(1, 1, 2), one(10, -1).reshape(1, 2, 1), "silu")
    h = 2.0 / (1 + np.exp(-2.0)) * 3.0
    assert (a.item(), b.item()) == (2.0, 3.0) and np.allclose(y.ravel(), [10 * h, -h])


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gradients_against_differences(kind):
    rng = np.random.default_rng(2)
    n, T, D, F = 2, 3, 4, 5
    x, dy = rng.normal(size=(2, n, T, D))
    gate, up, down = rng.normal(size=(n, F, D)), rng.normal(size=(n, F, D)), rng.normal(size=(n, D, F))
    _, a, b = orc.gated_ff(x, gate, up, down, kind)
    grads = orc.gated_ff_grad(dy, x, a, b, gate, up, down, kind)
    e = 1e-6
    for which, array in enumerate((x, gate, up, down)):
        for _ in range(6):
            at = tuple(rng.integers(k) for k in array.shape)
            was = array[at]
            f = []
            for s in (e, -e):
                array[at] = was + s
                f.append((dy * orc.gated_ff(x, gate, up, down, kind)[0]).sum())
            array[at] = was
            assert abs((f[0] - f[1]) / (2 * e) - grads[which][at]) < 1e-6


def test_orthogonalised_updates_by_singular_values():
    rng = np.random.default_rng(5)
    for rows, cols in ((3, 7), (7, 3), (4, 4), (1, 5)):
        g = rng.normal(size=(2, rows, cols))
        out, v = orc.orthogonalize(g, None, 0.0, False, 2, (1.5, -0.5, 0.25), 0.0, 2.0)
        assert v is None
        for m, o in zip(g, out):
            P, s, Q = np.linalg.svd(m, full_matrices=False)
            s = s / np.sqrt((s * s).sum())
            for _ in range(2):
                s = 1.5 * s - 0.5 * s ** 3 + 0.25 * s ** 5
            assert np.allclose(o, 2.0 * (P * s) @ Q, atol=1e-12)
    g, v = rng.normal(size=(2, 1, 3, 4))
    for nesterov in (False, True):
        out, w = orc.orthogonalize(g, v, 0.9, nesterov, 0, (1, 0, 0), 0.5, 1.0)
        u = g + 0.9 * w if nesterov else w
        assert np.allclose(w, 0.9 * v + g) and np.allclose(out, u / (np.sqrt((u * u).sum()) + 0.5))
