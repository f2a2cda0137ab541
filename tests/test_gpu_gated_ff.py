"""The gated feed-forward block on the GPU against the float64 oracle, through the C ABI.

Tolerances, from include/gpga.h's account of the pieces.  Two pieces of an operand are off by 2^-22 of its value, one by 2^-11, and what
falls below fp16's subnormals by 2^-39 of the largest value that shares the scale (2^-25 where that is 2^14 at least); two pieces each leave
out 2^-22 of a term; fp32 sums of K terms are off by (K + 16) 2^-24 of the terms' magnitudes.  A result is rounded once to the
activations' type, half a step of it, u = eps / 2 = 2^-24, 2^-8, 2^-11
relative.  Activation functions in fp32 are good to 2^-20 of |v|.  The bounds of rows of h and
[da | db] that stand in for their largest values are those of the formulas: |x| max|w| in 2-norms, squared; sum |dy| max|w| max(1.14 |b|, |a|).
"""
import numpy as np
import pytest

from oracle import matrix_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, 2.0 ** -24, 0.0), "bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}
E32, FN, FLOOR = 2.0 ** -24, 2.0 ** -20, 2.0 ** -39
ONE, TWO = 2.0 ** -11, 2.0 ** -22


@pytest.fixture(scope="module")
def hx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2105_09080_amd import harness
    return harness


def host(t):
    return t.detach().double().cpu().numpy()


def rows(rng, shape, dtype, pad=0, scale=1.0):
    """An (n, T, D) device tensor whose rows lie D + pad elements apart."""
    n, T, D = shape
    t = torch.zeros((n, T, D + pad), dtype=dtype, device="cuda")
    t[..., :D] = torch.as_tensor(rng.normal(size=shape) * scale).to(dtype).cuda()
    return t[..., :D]


def close(got, want, tol, what):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert np.isfinite(got).all(), f"{what}: not finite"
    off = np.abs(got - want) - tol
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max():.3e} over the tolerance {np.broadcast_to(tol, off.shape).flat[np.argmax(off)]:.3e} at {np.argmax(off)}"


def make(hx, n, D, F, off, seed, order=(0, 1, 2), **kw):
    """A simulation whose three matrices lie behind `off` other columns in the given order, and 3 more behind."""
    rng = np.random.default_rng(seed)
    d = off + 3 * D * F + 3
    X = rng.normal(size=(n, d)).astype(np.float32)
    at = [off + order.index(k) * D * F for k in range(3)]
    for k, width in ((0, D), (1, D), (2, F)):
        X[:, at[k]:at[k] + D * F] /= np.float32(np.sqrt(width))
    sim = hx.Simulation(n, d, topology="ring", H=4, lr=0.1, ld=d + 2, **kw)
    sim.set_state(X=X)
    gate, up = (X[:, at[k]:at[k] + D * F].reshape(n, F, D).astype(np.float64) for k in (0, 1))
    return sim, at, gate, up, X[:, at[2]:at[2] + D * F].reshape(n, D, F).astype(np.float64), rng


def norm(v, axis):
    return np.sqrt((v * v).sum(axis=axis))


def t(v):
    return v.transpose(0, 2, 1)


def forward_tolerances(x, gate, up, down, kind, dtype):
    """(tolerance of y, of a, of b) before the rounding to the type."""
    D, F = x.shape[2], gate.shape[1]
    ex, ew = {"f32": (TWO, TWO + TWO), "bf16": (0.0, ONE), "f16": (0.0, TWO)}[dtype]
    eh, ed = {"f32": (TWO, TWO + TWO), "bf16": (ONE, ONE), "f16": (ONE, TWO)}[dtype]
    y, a, b = orc.gated_ff(x, gate, up, down, kind)
    wide = lambda v: np.abs(v).max(axis=2, keepdims=True)
    ta, tb = ((ex + ew + (D + 16) * E32) * (np.abs(x) @ t(np.abs(w))) + FLOOR * (wide(x) * np.abs(w).sum(axis=2)[:, None, :] +
              np.abs(x).sum(axis=2, keepdims=True) * t(wide(w))) for w in (gate, up))
    value = orc.activation(kind, a)[0]
    bound = (norm(x, 2) * np.maximum(norm(gate, 2).max(axis=1), norm(up, 2).max(axis=1))[:, None]) ** 2
    th = 1.13 * ta * (np.abs(b) + tb) + np.abs(value) * tb + FN * np.abs(a * b) + eh * np.abs(value * b) + FLOOR * bound[..., None]
    ty = th @ t(np.abs(down)) + (ed + (F + 16) * E32) * (np.abs(value * b) @ t(np.abs(down))) + FLOOR * np.abs(value * b).sum(axis=2, keepdims=True) * t(wide(down))
    return (y, a, b), (ty, ta, tb)


def backward_tolerances(dy, x, a, b, gate, up, down, kind, dtype):
    T, D, F = x.shape[1], x.shape[2], gate.shape[1]
    f32 = dtype == "f32"
    value, slope = orc.activation(kind, a)
    m = np.abs(dy) @ np.abs(down)                       # magnitudes of dh's terms
    most = np.abs(dy).sum(axis=2) * np.abs(down).max(axis=(1, 2))[:, None]
    td = ((3 if f32 else 1) * TWO + (D + 16) * E32) * m + 2 * FLOOR * most[..., None]
    am, bm = np.abs(a).max(axis=2), np.abs(b).max(axis=2)
    floor = 2 * FLOOR * (most * np.maximum(1.14 * bm, am))[..., None]
    dh = np.abs(dy @ down)
    tda = td * np.abs(b * slope) + (4 * FN + TWO) * dh * np.abs(b) * (1 + np.abs(a)) + floor
    tdb = td * np.abs(value) + (FN + TWO) * dh * np.abs(a) + floor
    th = (FN + TWO) * np.abs(a * b) + 2 * FLOOR * (am * bm)[..., None]
    da, db, h = dh * np.abs(b * slope), dh * np.abs(value), np.abs(value * b)
    px = {"f32": 4 * TWO, "bf16": 2 * ONE, "f16": ONE + TWO}[dtype]
    big = np.maximum(np.abs(gate).max(axis=(1, 2)), np.abs(up).max(axis=(1, 2)))[:, None, None]
    tdx = tda @ np.abs(gate) + tdb @ np.abs(up) + (px + (2 * F + 16) * E32) * (da @ np.abs(gate) + db @ np.abs(up)) + FLOOR * big * (da + db).sum(axis=2, keepdims=True)
    # over tokens: the other operand is exact (two pieces with fp32), but for what falls below the subnormals of the node's scale
    po = (3 * TWO if f32 else TWO) + (T + 16) * E32
    low_x = FLOOR * (np.abs(x).max(axis=2) * most * np.maximum(1.14 * bm, am)).max(axis=1)[:, None, None] * 2 * T
    low_y = FLOOR * (np.abs(dy).max(axis=2) * am * bm).max(axis=1)[:, None, None] * 2 * T
    grads = [t(q) @ np.abs(x) + po * (t(v) @ np.abs(x)) + low_x for q, v in ((tda, da), (tdb, db))]
    grads.append(t(np.abs(dy)) @ th + po * (t(np.abs(dy)) @ h) + low_y)
    return tdx, grads


SIZES = [  # n, T, D, F, off, padding of the rows, order of the matrices
    (1, 1, 1, 1, 0, 0, (0, 1, 2)), (2, 5, 7, 9, 3, 1, (2, 0, 1)), (3, 33, 64, 64, 0, 0, (0, 1, 2)), (2, 70, 130, 257, 5, 3, (1, 2, 0)),
    (1, 300, 257, 100, 1, 0, (0, 1, 2)), (5, 64, 8, 600, 2, 8, (0, 2, 1)), (2, 65, 200, 3, 0, 0, (0, 1, 2)), (1, 2, 900, 31, 7, 5, (2, 1, 0)),
    (64, 260, 40, 520, 0, 0, (0, 1, 2)), (20, 1, 33, 65, 1, 0, (0, 1, 2)), (3, 12, 100, 130, 0, 4, (0, 1, 2)), (2, 129, 520, 64, 4, 0, (0, 1, 2)),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("n,T,D,F,off,pad,order", SIZES)
def test_forward_and_backward(hx, n, T, D, F, off, pad, order, kind, dtype):
    dt, u, sub = TYPES[dtype]
    sim, at, gate, up, down, rng = make(hx, n, D, F, off, T + D + F, order)
    x = rows(rng, (n, T, D), dt, pad)
    y, hidden = sim.gated_ff(x, *at, F, act=kind, keep=True)
    (wy, wa, wb), (ty, ta, tb) = forward_tolerances(host(x), gate, up, down, kind, dtype)
    close(y, wy, ty + u * (np.abs(wy) + ty) + sub, "y")
    close(hidden[..., :F], wa, ta + u * (np.abs(wa) + ta) + sub, "a")
    close(hidden[..., F:], wb, tb + u * (np.abs(wb) + tb) + sub, "b")
    alone, none = sim.gated_ff(x, *at, F, act=kind)
    assert none is None and torch.equal(alone, y)

    dy = rows(rng, (n, T, D), dt, pad, scale=0.1)
    a, b = host(hidden[..., :F]), host(hidden[..., F:])
    before = rng.normal(size=sim.G.shape).astype(np.float32)
    want = orc.gated_ff_grad(host(dy), host(x), a, b, gate, up, down, kind)
    tdx, tg = backward_tolerances(host(dy), host(x), a, b, gate, up, down, kind, dtype)
    for accumulate in (False, True):
        sim.set_state(G=before)
        dx = sim.gated_ff_grad(dy, x, hidden, *at, act=kind, accumulate=accumulate)
        close(dx, want[0], tdx + u * (np.abs(want[0]) + tdx) + sub, "dx")
        got = host(sim.G)
        left = np.ones(got.shape[1], dtype=bool)
        for k in range(3):
            block = slice(at[k], at[k] + D * F)
            had = before[:, block].astype(np.float64) * accumulate
            w = want[k + 1].reshape(n, -1)
            close(got[:, block], had + w, tg[k].reshape(n, -1) + 2 * E32 * (np.abs(had) + np.abs(w)), f"gradient {k}, accumulate={accumulate}")
            left[block] = False
        assert np.array_equal(got[:, left], before[:, left].astype(np.float64))
    again = sim.gated_ff_grad(dy, x, hidden, *at, act=kind, accumulate=False)
    assert torch.equal(again, dx)
    sim.close()
