"""The oracle of the language-model operators against differences of its own forward passes and against hand-made cases."""
import numpy as np
import pytest

from oracle import token_oracle as orc


def _slope(f, x, direction, h=1e-6):
    """Central difference of the scalar f along `direction`."""
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_embedding_gradient_is_that_of_the_lookup():
    rng = np.random.default_rng(0)
    n, V, D, T, scale = 2, 5, 3, 7, 1.7
    tokens = np.array([[0, 1, 1, -1, 4, 1, 0], [2, 2, 2, 2, 2, 2, 2]])
    E, w, step = rng.normal(size=(n, V, D)), rng.normal(size=(n, T, D)), rng.normal(size=(n, V, D))
    f = lambda e: (orc.embed(e, tokens, scale) * w).sum()
    g, _, count = orc.embed_grad(tokens, w, V, scale)
    assert (g * step).sum() == pytest.approx(_slope(f, E, step), rel=1e-8)
    assert count[0, 1, 0] == 3 and (g[0, 3] == 0).all() and count[0].sum() == 6


def test_embedding_of_padding_and_of_tokens_out_of_range():
    E = np.ones((1, 2, 2))
    y = orc.embed(E, np.array([[-1, 1, 2]]), 3.0)
    assert (y[0, 0] == 0).all() and (y[0, 1] == 3).all() and np.isnan(y[0, 2]).all()
    assert np.isnan(orc.embed_grad(np.array([[0, 2]]), np.ones((1, 2, 2)), 2, 1.0)[0]).all()


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_dropout_keeps_the_share_it_says_and_the_mean(p):
    n, T, D = 3, 64, 333
    keep, factor = orc.dropout_keep(n, T, D, p, seed=0x123456789ABCDEF, layer=3, k=17)
    share = keep.mean()
    assert abs(share - (1 - p)) < 5 * np.sqrt(p * (1 - p) / keep.size) + 2 ** -17
    assert factor == pytest.approx(1 / (1 - p), rel=2e-4)
    other = [orc.dropout_keep(n, T, D, p, seed=0x123456789ABCDEF, layer=l, k=k)[0] for l, k in ((4, 17), (3, 18))]
    for m in other:                                            # other layers and iterations: independent masks
        assert abs((m == keep).mean() - (p * p + (1 - p) ** 2)) < 5e-3
    assert not np.array_equal(keep[0], keep[1])


def test_layer_norm_gradients_are_those_of_the_forward_pass():
    rng = np.random.default_rng(1)
    n, T, D, eps = 2, 3, 9, 1e-3
    u, w, gamma, beta = rng.normal(size=(n, T, D)), rng.normal(size=(n, T, D)), rng.normal(size=(n, D)), rng.normal(size=(n, D))
    _, mean, rstd = orc.layer_norm(u, gamma, beta, eps)
    du, dg, db = orc.layer_norm_grad(w, u, mean, rstd, gamma)
    su, sg = rng.normal(size=u.shape), rng.normal(size=gamma.shape)
    assert (du * su).sum() == pytest.approx(_slope(lambda v: (orc.layer_norm(v, gamma, beta, eps)[0] * w).sum(), u, su), rel=1e-6)
    assert (dg * sg).sum() == pytest.approx(_slope(lambda v: (orc.layer_norm(u, v, beta, eps)[0] * w).sum(), gamma, sg), rel=1e-6)
    assert (db * sg).sum() == pytest.approx(_slope(lambda v: (orc.layer_norm(u, gamma, v, eps)[0] * w).sum(), beta, sg), rel=1e-6)


def test_token_loss_gradient_and_rows_that_do_not_count():
    rng = np.random.default_rng(2)
    n, T, V = 2, 4, 6
    z, step = rng.normal(size=(n, T, V)), rng.normal(size=(n, T, V))
    labels = np.array([[1, -1, 5, 0], [-1, -1, -1, -1]])
    loss, dz = orc.token_loss(z, labels, grad_scale=3.0)
    assert (dz[0] * step[0]).sum() / 3.0 == pytest.approx(_slope(lambda v: orc.token_loss(v, labels)[0][0], z, step), rel=1e-6)
    assert loss[1] == 0 and (dz[1] == 0).all() and (dz[0, 1] == 0).all()
    assert orc.token_loss(np.zeros((1, 2, V)), np.array([[0, 3]]))[0][0] == pytest.approx(np.log(V))


def test_token_loss_of_large_logits_keeps_its_digits():
    z = np.array([[[1e4, 1e4 - 1.0, -np.inf]]])
    assert orc.token_loss(z, np.array([[1]]))[0][0] == pytest.approx(np.log1p(np.exp(-1.0)) + 1.0, rel=1e-12)
    assert np.isinf(orc.token_loss(z, np.array([[2]]))[0][0])
    assert np.isnan(orc.token_loss(np.full((1, 1, 3), -np.inf), np.array([[0]]))[0][0])
