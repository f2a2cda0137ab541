"""The gated feed-forward block on matrices, rows and kept values of very different sizes, against the float64 oracle.  64 tokens of a node go
through one kernel and 65 through others; both have to be right.

Tolerances are taken from the terms that make up a result, each with its own size, and from no bound over several of them.  With e for
the pieces of an operand (2^-22 for two, 2^-11 for one, 0 where one is exact), a sum of K terms p_k q_k is off by
(e + (sqrt K + 16) 2^-24) times the sum of |p_k q_k|, or |p| |q| in 2-norms, which is more: K roundings of fp32 that go up as often as down, each
of a partial sum of at most that.
What falls below fp16's subnormals is 2^-39 of the largest value that shares the scale, 2^-40 where that is a power of two above it.  Errors of the elements of a
vector are independent, so a product takes them by the root of the sum of their squares.  Rounding to the activations' type: u = eps / 2.
"""
import numpy as np
import pytest

from oracle import matrix_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}
E32, FN, FLOOR, ONE, TWO = 2.0 ** -24, 2.0 ** -20, 2.0 ** -39, 2.0 ** -11, 2.0 ** -22
N, D, F = 2, 72, 90


@pytest.fixture(scope="module")
def hx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2105_09080_amd import harness
    return harness


def norm(v, axis):
    return np.sqrt((v * v).sum(axis=axis))


def t(v):
    return v.transpose(0, 2, 1)


def sums(k):
    return (np.sqrt(k) + 16) * E32


def spread_matrices(kind, rng):
    gate, up, down = rng.normal(size=(N, F, D)) / np.sqrt(D), rng.normal(size=(N, F, D)) / np.sqrt(D), rng.normal(size=(N, D, F)) / np.sqrt(F)
    if kind == "up small":
        up *= 1e-6
    if kind == "gate small":
        gate *= 1e-6
    if kind == "one gate row":
        gate[:, 5] *= 1e4
    if kind == "one up row":
        up[:, 5] *= 1e4
    if kind == "apart":                                              # neither has the other's size
        gate *= 2.0 ** -60
        up *= 2.0 ** 60
    if kind == "huge":
        gate *= 2.0 ** 55
        up *= 2.0 ** 55
    if kind == "tiny":
        gate *= 2.0 ** -52
        up *= 2.0 ** -52
    if kind == "every row":                                          # rows from 2^-30 to 2^30, and the columns that they meet
        s = 2.0 ** np.linspace(-30, 30, F).round()
        rng.shuffle(s)
        up *= s[None, :, None]
        down /= s[None, None, :]
    if kind == "zero rows":
        gate[:, ::3] = 0.0
        up[:, 1::3] = 0.0
        up[0] *= 1e-6
    return [w.astype(np.float32).astype(np.float64) for w in (gate, up, down)]


def make(hx, gate, up, down):
    sim = hx.Simulation(N, 3 * D * F, topology="ring", H=4, lr=0.1)
    sim.set_state(X=np.concatenate([w.reshape(N, -1) for w in (gate, up, down)], axis=1).astype(np.float32))
    return sim, (0, D * F, 2 * D * F)


def activations(rng, shape, dt, scale=1.0):
    v = torch.as_tensor(rng.normal(size=shape) * scale).to(dt).cuda()
    return v, v.double().cpu().numpy()


def forward_tolerances(x, gate, up, down, kind, dtype):
    """(y, a, b) and how far they may be off: of y the 2-norm of a token's error, of a and b each element's."""
    ex, ew = {"f32": (TWO, TWO + TWO), "bf16": (0.0, ONE), "f16": (0.0, TWO)}[dtype]
    eh, ed = {"f32": (TWO, TWO + TWO), "bf16": (ONE, ONE), "f16": (ONE, TWO)}[dtype]
    y, a, b = orc.gated_ff(x, gate, up, down, kind)
    xn = norm(x, 2)[..., None]
    ta, tb = ((ex + ew + sums(D)) * xn * norm(w, 2)[:, None, :] for w in (gate, up))
    value = orc.activation(kind, a)[0]
    tv = np.maximum(np.abs(orc.activation(kind, a + ta)[0] - value), np.abs(orc.activation(kind, a - ta)[0] - value)) + FN * np.abs(a)
    h, size = value * b, (norm(gate, 2) * norm(up, 2))[:, None, :]
    # the bound of an element of h is up to 2^3 above |x|^2 |wg_f| |wu_f|; that of one of the down matrix's row 2^2 above the largest of them
    th = tv * (np.abs(b) + tb) + np.abs(value) * tb + eh * np.abs(h) + 8 * FLOOR * xn ** 2 * size
    most = (np.abs(down) * size).max(axis=2)                         # n, D
    low = 4 * FLOOR * np.einsum("ntf,nd->ntd", np.abs(h) / np.where(size > 0, size, 1.0), most)
    ty = np.sqrt((th ** 2) @ t(down ** 2)) + (ed + sums(F)) * (np.abs(h) @ t(np.abs(down))) + low
    return (y, a, b), (norm(ty, 2), ta, tb)


MATRICES = ["alike", "up small", "gate small", "one gate row", "one up row", "apart", "every row", "zero rows", "huge", "tiny"]


def with_types(kinds, not_fp16):
    """(kind, type), without those whose values are not in fp16's range."""
    return [(k, d) for k in kinds for d in TYPES if d != "f16" or k not in not_fp16]


@pytest.mark.parametrize("kind,dtype", with_types(MATRICES, ("apart", "every row", "huge", "tiny")))
@pytest.mark.parametrize("T", [64, 65])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_forward(hx, kind, act, T, dtype):
    dt, u = TYPES[dtype]
    rng = np.random.default_rng(len(kind) + T)
    gate, up, down = spread_matrices(kind, rng)
    sim, at = make(hx, gate, up, down)
    x, xd = activations(rng, (N, T, D), dt)
    y, hidden = sim.gated_ff(x, *at, F, act=act, keep=True)
    with np.errstate(over="ignore", invalid="ignore"):
        (wy, wa, wb), (ty, ta, tb) = forward_tolerances(xd, gate, up, down, act, dtype)
    sub = 2.0 ** -25 if dtype == "f16" else 0.0                       # below fp16's smallest normal numbers
    hidden, y = hidden.double().cpu().numpy(), y.double().cpu().numpy()
    assert (np.abs(hidden[..., :F] - wa) <= ta + u * (np.abs(wa) + ta) + sub).all()
    assert (np.abs(hidden[..., F:] - wb) <= tb + u * (np.abs(wb) + tb) + sub).all()
    off, tol = norm(y - wy, 2), ty * (1 + u) + u * norm(wy, 2) + sub * np.sqrt(D)
    if dtype == "f32":
        # the tolerance tells.  A row 10^4 above the others has a's error of (2^-20 + 25 2^-24) |x| |w| = 2.4e-6 * 8.5 * 10^4 = 0.2, and tokens where it
        # is not the whole result (a large and negative) or all of it (large) are few enough for y's median to be off by 10^-4 or so
        far = float(np.median(ty / norm(wy, 2)))
        assert far < (1e-3 if kind.startswith("one") else 1e-4), far
    worst = float((off / norm(wy, 2)).max())
    assert (off <= tol).all(), worst
    sim.close()


def backward_tolerances(dy, x, a, b, gate, up, down, kind, dtype):
    """dx and the matrices' gradients, and how far they may be off: 2-norms of dx's tokens and of the gradients' matrices."""
    T = x.shape[1]
    f32 = dtype == "f32"
    value, slope = orc.activation(kind, a)
    dh = dy @ down
    # dh: dy exact but with fp32, the matrix in two pieces by rows; dh's bound is the sum of |dy| max |row|
    wide = np.abs(down).max(axis=2)
    th = ((3 if f32 else 1) * TWO + sums(D)) * (np.abs(dy) @ np.abs(down)) + 2 * FLOOR * D * (np.abs(dy) * wide[:, None, :]).max(axis=2)[..., None]
    most = (np.abs(dy) * wide[:, None, :]).sum(axis=2)[..., None]
    vm, bm = np.abs(value).max(axis=2)[..., None], np.abs(b).max(axis=2)[..., None]
    # bounds: 1.14 for the slope, for act(a) a where it is positive and at most 2^2 too much where all are not; powers of two above them
    near = np.where(np.abs(a) < 40, np.abs(a), 1.0)                  # act is good to 2^-20 of it, its slope to 2^-18; beyond, a or nothing
    tda = th * np.abs(b * slope) + (4 * FN * (1 + near) + TWO) * np.abs(dh * b) + 4 * FLOOR * most * bm
    tdb = th * np.abs(value) + TWO * np.abs(dh * value) + FN * np.abs(dh) * near + 8 * FLOOR * most * vm
    thh = TWO * np.abs(value * b) + FN * np.abs(b) * near + 8 * FLOOR * vm * bm
    da, db, h = dh * b * slope, dh * value, value * b
    want = [da @ gate + db @ up, t(da) @ x, t(db) @ x, t(dy) @ h]
    # of dx: pieces of da, db and of the matrices, each by a scale of the whole matrix
    px = {"f32": 4 * TWO, "bf16": 2 * ONE, "f16": ONE + TWO}[dtype]
    root = lambda v, w: np.sqrt((v ** 2) @ (w ** 2))
    tdx = root(tda, gate) + root(tdb, up) + px * (root(da, gate) + root(db, up)) + sums(2 * F) * (np.abs(da) @ np.abs(gate) + np.abs(db) @ np.abs(up))
    for v, w in ((da, gate), (db, up)):
        tdx = tdx + 2 * FLOOR * np.abs(w).max(axis=(1, 2))[:, None, None] * norm(v, 2)[..., None]
    po = (3 * TWO if f32 else TWO) + sums(T)
    tol = [norm(tdx, 2)]
    for tv, v, w, bound in ((tda, da, x, most * bm), (tdb, db, x, most * vm), (thh, h, dy, vm * bm)):
        # the other operand is exact (two pieces with fp32), but for what falls below the subnormals of the node's scale
        low = 8 * FLOOR * (np.abs(w).max(axis=2)[..., None] * bound).max(axis=1)[..., None] / np.where(bound > 0, bound, 1.0)
        e = root(t(tv), np.abs(w)) + po * (t(np.abs(v)) @ np.abs(w)) + root(t(np.abs(v)), low * np.ones_like(w))
        tol.append(np.sqrt((e ** 2).sum(axis=(1, 2))))
    return want, tol


KEPT = ["alike", "b small", "a small", "a large and negative", "up small", "gate small", "one gate row", "one up row", "apart", "column", "zero rows", "no b", "no a", "no gate",
        "b far", "a far"]


@pytest.mark.parametrize("kind,dtype", with_types(KEPT, ("apart", "column", "b far", "a far")))
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [7, 130])
def test_backward(hx, kind, T, act, dtype):
    """The kept [a | b] of one token, or of all, may be of any size beside each other, as the matrices may."""
    dt, u = TYPES[dtype]
    rng = np.random.default_rng(len(kind) + T)
    gate, up, down = spread_matrices(kind, rng)
    if kind == "column":                                             # a column of x that gate sees and up does not
        up[:, :, 3] = 0.0
    if kind == "no gate":
        gate[:] = 0.0
    sim, at = make(hx, gate, up, down)
    x, xd = activations(rng, (N, T, D), dt)
    if kind == "column":
        x[..., 3] *= 2.0 ** 20
        xd = x.double().cpu().numpy()
    dy, dyd = activations(rng, (N, T, D), dt, 2.0 ** -5)
    _, a, b = orc.gated_ff(xd, gate, up, down, act)
    if kind == "b small":
        b *= 2.0 ** -20
    if kind == "b far":
        b *= 2.0 ** -100
    if kind == "a far":
        a *= 2.0 ** -60
    if kind == "a small":
        a *= 2.0 ** -14
        a[:, 1] *= 2.0 ** 20                                         # and a token where it is not
    if kind == "a large and negative":                              # where act(a) and its slope are nothing
        a[..., ::2] = -2.0 ** 15
    if kind == "no b":
        b[:] = 0.0
    if kind == "no a":
        a[:] = 0.0
    hidden = torch.as_tensor(np.concatenate([a, b], axis=2)).to(dt).cuda()
    kept = hidden.double().cpu().numpy()
    a, b = kept[..., :F], kept[..., F:]
    with np.errstate(over="ignore"):
        want, tol = backward_tolerances(dyd, xd, a, b, gate, up, down, act, dtype)
    dx = sim.gated_ff_grad(dy, x, hidden, *at, act=act).double().cpu().numpy()
    sub = 2.0 ** -25 * np.sqrt(D) if dtype == "f16" else 0.0
    off, size = norm(dx - want[0], 2), norm(want[0], 2)
    if dtype == "f32" and kind != "no gate" and size.any():
        far = float(np.median(tol[0] / np.maximum(size, 1e-300)))
        assert far < 1e-3, far
    worst = float((off / np.maximum(size, 1e-300)).max())
    assert (off <= tol[0] * (1 + u) + u * size + sub).all(), worst
    G = sim.G.double().cpu().numpy()
    for k in range(3):
        got = G[:, at[k]:at[k] + D * F].reshape(want[k + 1].shape)
        size = np.sqrt((want[k + 1] ** 2).sum(axis=(1, 2)))
        off = np.sqrt(((got - want[k + 1]) ** 2).sum(axis=(1, 2)))
        if size.all():
            far = float((tol[k + 1] / size).max())
            assert far < 1e-3, (k, far)
        assert (off <= tol[k + 1] + E32 * size).all(), (k, float((off / np.maximum(size, 1e-300)).max()), float((tol[k + 1] / np.maximum(size, 1e-300)).max()))
    sim.close()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,T,D", [(3, 2000, 64), (8, 4096, 320), (200, 70, 64)])
def test_both_pieces_of_every_h(hx, n, T, D, act):
    """Diagonal matrices: y_j = act(g_j x_j) (u_j x_j) w_j, every element by itself: some twenty roundings to 2^-22 and of fp32 and an act that is good
    to 2^-20 of a, 2^-16 of |a| |b| |w| together, and what falls below the subnormals of |x|^2.  A second piece that does not go with the first
    leaves 2^-11."""
    rng = np.random.default_rng(T)
    g, u, w = (rng.uniform(0.5, 2.0, size=(3, n, D))).astype(np.float32).astype(np.float64)
    sim = hx.Simulation(n, 3 * D * D, topology="ring", H=4, lr=0.1)
    X = torch.zeros((n, 3, D, D), device="cuda")
    for k, v in enumerate((g, u, w)):
        X[:, k].diagonal(dim1=1, dim2=2).copy_(torch.as_tensor(v).cuda())
    sim.X.copy_(X.view(n, -1))
    x, xd = activations(rng, (n, T, D), torch.float32, 2.0)
    y = sim.gated_ff(x, 0, D * D, 2 * D * D, D, act=act)[0].double()
    sim.close()
    gt, ut, wt, xt = (torch.as_tensor(v).cuda() for v in (g[:, None], u[:, None], w[:, None], xd))
    a, b = gt * xt, ut * xt
    want = (a * torch.sigmoid(a) if act == "silu" else a * torch.special.ndtr(a)) * b * wt
    tol = 2.0 ** -16 * (torch.where(a < 0, a.abs().clamp(max=1.0), a) * b * wt).abs() * torch.where(a < 0, 2.0 ** -3, 1.0)
    tol = tol + 2.0 ** -19 * (b * wt).abs() * (a < 0) + 2.0 ** -34 * xt.square().sum(dim=2, keepdim=True) * 8
    bad = (y - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((y - want).abs() / tol).max()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,D,F", [(300, 64, 128), (40, 512, 640), (2, 2048, 2048)])
def test_both_pieces_of_every_da(hx, n, D, F, act):
    """One token a node: the matrices' gradients are products of one da_f, db_f or h_f and one x_j or dy_j, every element by itself.  dy has one element
    other than 0, so dh_f = dy_j Wd_jf."""
    rng = np.random.default_rng(D)
    sim = hx.Simulation(n, 3 * D * F, topology="ring", H=4, lr=0.1)
    sim.X.normal_()
    down = sim.X[:, 2 * D * F:].view(n, D, F)[:, 5].double()
    x, _ = activations(rng, (n, 1, D), torch.float32)
    dy = torch.zeros((n, 1, D), device="cuda")
    dy[:, 0, 5] = torch.as_tensor(rng.uniform(0.5, 2.0, size=n).astype(np.float32)).cuda()
    hidden, _ = activations(rng, (n, 1, 2 * F), torch.float32)
    sim.gated_ff_grad(dy, x, hidden, 0, D * F, 2 * D * F, act=act)
    a, b = hidden[:, 0, :F].double(), hidden[:, 0, F:].double()
    s = torch.sigmoid(a) if act == "silu" else torch.special.ndtr(a)
    slope = s + a * s * (1 - s) if act == "silu" else s + a * torch.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    dh, xs = dy[:, 0, 5].double()[:, None] * down, x[:, 0].double()
    rest = {"da": (dh * b * slope, 2.0 ** -17 * (dh * b).abs()), "db": (dh * a * s, 2.0 ** -17 * dh.abs() * a.abs().clamp(min=0.1))}
    for k, name in enumerate(rest):
        v, tol = rest[name]
        got = sim.G[:, k * D * F:(k + 1) * D * F].view(n, F, D).double()
        # the bound of da is some 2^6 above it, x's scale its largest value: 2^-39 of either
        most = v.abs().amax(dim=1, keepdim=True) * 2.0 ** -31
        off = (got - v[:, :, None] * xs[:, None]).abs() / ((tol + most)[:, :, None] * xs[:, None].abs() + v.abs()[:, :, None] * 2.0 ** -36)
        assert not (off > 1).any(), (name, int((off > 1).sum()), float(off.max()))
    h = a * s * b
    got = sim.G[:, 2 * D * F:].view(n, D, F)[:, 5].double()
    off = (got - h * dy[:, 0, 5].double()[:, None]).abs() / (2.0 ** -17 * (b.abs() * a.abs().clamp(min=0.1)) + h.abs().amax(dim=1, keepdim=True) * 2.0 ** -31) / dy[:, 0, 5].double()[:, None]
    assert not (off > 1).any(), ("h", int((off > 1).sum()), float(off.max()))
    sim.close()
