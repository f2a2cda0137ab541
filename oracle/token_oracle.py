"""CPU oracle for the language-model operators (TEST INFRASTRUCTURE ONLY): plain float64 NumPy statements of the
formulas in include/gpga.h, one node and one token at a time where that is the clearest.  Parameters come as float32
arrays, activations as whatever values the device holds; nothing is rounded here.  Pinned by finite differences and by
hand-made cases in tests/test_oracle_token_pins.py."""
from __future__ import annotations

import numpy as np

from .gpga_oracle import philox4x32_10


def embed(table, tokens, scale):
    """table (n, V, D), tokens (n, T): (n, T, D)."""
    n, V, D = table.shape
    y = np.zeros((*tokens.shape, D))
    for i in range(n):
        for t, tok in enumerate(tokens[i]):
            if tok >= V:
                y[i, t] = np.nan
            elif tok >= 0:
                y[i, t] = scale * table[i, tok].astype(np.float64)
    return y


def embed_grad(tokens, dy, V, scale):
    """(gradient (n, V, D), sum of the terms' magnitudes, number of terms)."""
    n, T, D = dy.shape
    g, size, count = np.zeros((n, V, D)), np.zeros((n, V, D)), np.zeros((n, V, 1))
    for i in range(n):
        for t, tok in enumerate(tokens[i]):
            if 0 <= tok < V:
                g[i, tok] += scale * dy[i, t].astype(np.float64)
                size[i, tok] += abs(scale) * np.abs(dy[i, t].astype(np.float64))
                count[i, tok] += 1
        if (tokens[i] >= V).any():
            g[i] = np.nan
    return g, size, count


def dropout_keep(n, T, D, p, seed, layer, k):
    """(mask (n, T, D) of booleans, factor of what stays)."""
    drop = int(float(np.float32(p)) * 65536.0 + 0.5)
    octs = (D + 7) // 8
    keep = np.zeros((n, T, octs * 8), dtype=bool)
    group = np.arange(T * octs)
    for i in range(n):
        words = philox4x32_10(group, i, k & 0xFFFFFFFF, 4 + 256 * layer, seed & 0xFFFFFFFF, seed >> 32)
        lots = np.zeros((T * octs, 8), dtype=np.int64)
        for j in range(4):
            w = np.broadcast_to(np.asarray(words[j]), group.shape).astype(np.int64)
            lots[:, 2 * j], lots[:, 2 * j + 1] = w & 0xFFFF, w >> 16
        keep[i] = (lots >= drop).reshape(T, octs * 8)
    return keep[:, :, :D], 65536.0 / (65536 - drop)


def dropout(x, residual, p, seed, layer, k):
    x = x.astype(np.float64)
    if p > 0:
        keep, factor = dropout_keep(*x.shape, p, seed, layer, k)
        x = np.where(keep, x * factor, 0.0)
    return x if residual is None else x + residual.astype(np.float64)


def layer_norm(u, gamma, beta, eps):
    """u (n, T, D), gamma, beta (n, D): (y, mean, rstd)."""
    u = u.astype(np.float64)
    mean = u.mean(axis=2, keepdims=True)
    rstd = 1.0 / np.sqrt(((u - mean) ** 2).mean(axis=2, keepdims=True) + eps)
    return (u - mean) * rstd * gamma[:, None, :].astype(np.float64) + beta[:, None, :].astype(np.float64), mean[..., 0], rstd[..., 0]


def layer_norm_grad(dy, u, mean, rstd, gamma):
    """(du, dgamma, dbeta) for given statistics."""
    dy, u = dy.astype(np.float64), u.astype(np.float64)
    xh = (u - mean[..., None]) * rstd[..., None]
    h = dy * gamma[:, None, :].astype(np.float64)
    du = rstd[..., None] * (h - h.mean(axis=2, keepdims=True) - xh * (h * xh).mean(axis=2, keepdims=True))
    return du, (dy * xh).sum(axis=1), dy.sum(axis=1)


def token_loss(z, labels, grad_scale=1.0):
    """(loss (n,), dz (n, T, V))."""
    z = z.astype(np.float64)
    n, T, V = z.shape
    loss, dz = np.zeros(n), np.zeros_like(z)
    for i in range(n):
        counted = int((labels[i] >= 0).sum())
        for t in range(T):
            label = labels[i, t]
            if label < 0:
                continue
            if label >= V:
                loss[i], dz[i, t] = np.nan, np.nan
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                top = z[i, t].max()
                e = np.exp(z[i, t] - top)
                loss[i] += (np.log(e.sum()) + (top - z[i, t, label])) / counted
                dz[i, t] = e / e.sum()
            dz[i, t, label] -= 1.0
            dz[i, t] *= grad_scale / counted
    return loss, dz
