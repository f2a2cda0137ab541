"""Performance cases of the gated feed-forward block on the nodes' own parameters and of orthogonalised updates of their matrices.

Every node i has parameters of its own, a row of X; the operators read matrices there, row-major blocks at column offsets,
and find and leave their gradients in the same columns of G.  Activations are (n, T, D) tensors, T tokens a node.

  ff       a = x Wg_i^T, b = x Wu_i^T, y = (act(a) * b) Wd_i^T, with Wg_i, Wu_i of F x D and Wd_i of D x F; act is
           silu(v) = v / (1 + exp(-v)) or gelu(v) = v (1 + erf(v / sqrt 2)) / 2; for training [a | b] is kept, rounded
  ff_grad  from dy, x and the kept [a | b]: dx, and the gradients of the three matrices, summed over the tokens, into G (or
           added to what is there)
  orth     v <- mu v + g (where the caller keeps v), u = g + mu v (Nesterov) or v, X0 = u / (|u|_F + eps), five times
           X <- p X + q (X X^T) X + r (X X^T)^2 X (from the side with fewer rows), and scale * X takes g's place

Where `own` is false the same results come from elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_P, _Q, _R = 3.4445, -4.7750, 2.0315
_EPS = 1e-7
_MU = 0.95


def listed():
    return [
        # One new token on each of eight nodes, without gradients: every matrix is read once for one row.  Latency and bandwidth.
        dict(name="ff_next_token", op="ff", n=8, T=1, D=768, F=2048, dtype="bf16", act="silu", off=0, keep=False),
        # A handful of sequences answered side by side: few rows, still bound by the matrices.
        dict(name="ff_few_tokens", op="ff", n=4, T=24, D=1024, F=4096, dtype="f16", act="silu", off=0, keep=False),
        # The block in a training step: 8 sequences of 512 tokens on each of 8 nodes, what the backward pass needs is kept.
        dict(name="ff_batch", op="ff", n=8, T=4096, D=768, F=2048, dtype="bf16", act="silu", off=0, keep=True),
        # Sizes that no tile divides, in single precision, behind other layers' parameters.
        dict(name="ff_odd", op="ff", n=5, T=513, D=257, F=1023, dtype="f32", act="gelu", off=7, keep=True),
        # The largest: twice the tokens on a wider block, as in evaluation of long texts.
        dict(name="ff_large", op="ff", n=8, T=8192, D=1024, F=4096, dtype="bf16", act="gelu", off=0, keep=False),
        # The backward pass of the training step.
        dict(name="ff_grad_batch", op="ff_grad", n=8, T=4096, D=768, F=2048, dtype="bf16", act="silu", off=0, accumulate=False),
        # A matrix that is used twice in a model: its gradient is added to the other use's.  Odd everywhere, single precision.
        dict(name="ff_grad_odd", op="ff_grad", n=7, T=333, D=511, F=1021, dtype="f32", act="gelu", off=3, accumulate=True),
        # Two nodes with a wide block in half precision.
        dict(name="ff_grad_wide", op="ff_grad", n=2, T=2048, D=2048, F=5632, dtype="f16", act="silu", off=0, accumulate=False),
        # Small square matrices of twenty nodes: launches and their gaps.
        dict(name="orth_small", op="orth", n=20, rows=64, cols=64, count=1, off=0, velocity=False, nesterov=False),
        # The gate's and the up projection's updates of the block above, with momentum: two matrices of every node at once.
        dict(name="orth_gate_up", op="orth", n=8, rows=2048, cols=768, count=2, off=0, velocity=True, nesterov=True),
        # Square projections, several of a node side by side.
        dict(name="orth_square", op="orth", n=4, rows=1024, cols=1024, count=4, off=0, velocity=False, nesterov=False),
        # A wide matrix with odd sides.
        dict(name="orth_odd", op="orth", n=5, rows=257, cols=1023, count=1, off=5, velocity=True, nesterov=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' range; no pass computes more than the largest listed one of its operator."""
    op = rng.choice(["ff", "ff", "ff_grad", "ff_grad", "orth"])
    n = _log_int(rng, 1, 32)
    off = rng.choice([0, 0, 1, 8, 13])
    if op == "orth":
        rows, cols = _log_int(rng, 8, 2048), _log_int(rng, 8, 2048)
        small, wide = min(rows, cols), max(rows, cols)
        n = max(1, min(n, 19_000_000_000 // (small * small * wide)))
        count = max(1, min(rng.choice([1, 1, 2, 3]), 19_000_000_000 // (n * small * small * wide)))
        velocity = rng.random() < 0.5
        return dict(op=op, n=n, rows=rows, cols=cols, count=count, off=off, velocity=velocity,
                    nesterov=velocity and rng.random() < 0.5)
    D = _log_int(rng, 16, 2048)
    F = _log_int(rng, 16, 8192)
    n = max(1, min(n, (33_000_000 if op == "ff" else 20_000_000) // (D * F)))
    T = _log_int(rng, 1, 8192)
    most = 250_000_000_000 if op == "ff" else 50_000_000_000
    T = max(1, min(T, most // (n * D * F), 150_000_000 // (n * F)))
    c = dict(op=op, n=n, T=T, D=D, F=F, dtype=rng.choice(["f32", "bf16", "bf16", "f16"]), act=rng.choice(["silu", "gelu"]), off=off)
    return dict(c, keep=rng.random() < 0.6) if op == "ff" else dict(c, accumulate=rng.random() < 0.4)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _columns(case):
    """Parameters a node has: a block of `off` floats that belongs to other layers, then this one's."""
    if case["op"] == "orth":
        return case["off"] + case["count"] * case["rows"] * case["cols"]
    return case["off"] + 3 * case["D"] * case["F"]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(case, seed):
    g = _generator(seed)
    n, off = case["n"], case["off"]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=g) * scale

    if case["op"] == "orth":
        # what a backward pass leaves: a few directions that the tokens share, and noise in all others
        c, rows, cols = n * case["count"], case["rows"], case["cols"]
        k = min(6, rows, cols)
        strong = torch.bmm(normal(c, rows, k), normal(c, k, cols) * (0.5 ** torch.arange(k, device="cuda")).view(1, k, 1))
        s = dict(case=case, grad=(1e-3 * (0.3 * strong + normal(c, rows, cols))).view(n, -1))
        s["v"] = normal(n, case["count"] * rows * cols, scale=1e-2) if case["velocity"] else None
        return s
    T, D, F = case["T"], case["D"], case["F"]
    dtype = _DTYPE[case["dtype"]]
    X = normal(n, _columns(case))
    X[:, off:off + 2 * F * D] *= D ** -0.5
    X[:, off + 2 * F * D:] *= F ** -0.5
    s = dict(case=case, X=X, x=normal(n, T, D).to(dtype))
    if case["op"] == "ff_grad":
        s["dy"] = normal(n, T, D, scale=1e-2).to(dtype)
        s["hidden"] = normal(n, T, 2 * F).to(dtype)
        if case["accumulate"]:
            s["other"] = normal(n, 3 * D * F, scale=1e-2)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2105_09080_amd.harness import Simulation
        s["sim"] = Simulation(case["n"], _columns(case), topology="ring", H=6, lr=0.1)
        if "X" in s:
            s["sim"].X.copy_(s.pop("X"))
    return s


# ---- the operators in their plain form ----------------------------------------------------------------------------------

def _act(kind, v):
    return v / (1 + torch.exp(-v)) if kind == "silu" else 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))


def _act_grad(kind, v):
    if kind == "silu":
        q = 1 / (1 + torch.exp(-v))
        return q * (1 + v * (1 - q))
    return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))


def _matrices(s):
    case = s["case"]
    n, D, F, off = case["n"], case["D"], case["F"], case["off"]
    gate, up, down = s["X"][:, off:].split([F * D, F * D, D * F], dim=1)
    return gate.reshape(n, F, D), up.reshape(n, F, D), down.reshape(n, D, F)


def _step(x):
    a = torch.bmm(x, x.transpose(1, 2))
    return _P * x + torch.bmm(_Q * a + _R * torch.bmm(a, a), x)


def _plain_orth(s):
    case = s["case"]
    n, rows, cols = case["n"], case["rows"], case["cols"]
    u = s["grad"]
    if s["v"] is not None:
        s["v"].mul_(_MU).add_(u)
        u = u + _MU * s["v"] if case["nesterov"] else s["v"]
    u = u.view(n * case["count"], rows, cols)
    u = u / (u.square().sum(dim=(1, 2), keepdim=True).sqrt() + _EPS)
    tall = rows > cols
    x = u.transpose(1, 2).contiguous() if tall else u
    x = _step(_step(_step(_step(_step(x)))))
    x = (x.transpose(1, 2) if tall else x) * max(1.0, rows / cols) ** 0.5
    return {"update": x.reshape(n, -1), "v": s["v"]} if s["v"] is not None else {"update": x.reshape(n, -1)}


def _plain(s):
    case = s["case"]
    if case["op"] == "orth":
        return _plain_orth(s)
    n, F = case["n"], case["F"]
    dtype = _DTYPE[case["dtype"]]
    gate, up, down = _matrices(s)
    x = s["x"].float()
    if case["op"] == "ff":
        a, b = torch.bmm(x, gate.transpose(1, 2)), torch.bmm(x, up.transpose(1, 2))
        y = torch.bmm(_act(case["act"], a) * b, down.transpose(1, 2)).to(dtype)
        return {"y": y, "hidden": torch.cat([a, b], dim=2).to(dtype)} if case["keep"] else {"y": y}
    dy = s["dy"].float()
    a, b = s["hidden"][..., :F].float(), s["hidden"][..., F:].float()
    value = _act(case["act"], a)
    dh = torch.bmm(dy, down)
    da, db = dh * b * _act_grad(case["act"], a), dh * value
    dx = torch.bmm(da, gate) + torch.bmm(db, up)
    grads = [torch.bmm(da.transpose(1, 2), x), torch.bmm(db.transpose(1, 2), x), torch.bmm(dy.transpose(1, 2), value * b)]
    out = torch.cat([w.reshape(n, -1) for w in grads], dim=1)
    return {"dx": dx.to(dtype), "grads": s["other"] + out if case["accumulate"] else out}


# ---- the framework's calls ------------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    case, sim = s["case"], s["sim"]
    off = case["off"]
    block = sim.G[:, off:]
    if case["op"] == "orth":
        block.copy_(s["grad"])  # the backward pass leaves it there
        sim.orthogonalize(off, case["rows"], case["cols"], count=case["count"], velocity=s["v"],
                          mu=_MU if case["velocity"] else 0.0, nesterov=case["nesterov"], steps=5, coefficients=(_P, _Q, _R),
                          eps=_EPS, scale=max(1.0, case["rows"] / case["cols"]) ** 0.5)
        return {"update": block, "v": s["v"]} if s["v"] is not None else {"update": block}
    D, F = case["D"], case["F"]
    columns = (off, off + F * D, off + 2 * F * D)
    if case["op"] == "ff":
        y, hidden = sim.gated_ff(s["x"], *columns, F, act=case["act"], keep=case["keep"])
        return {"y": y, "hidden": hidden} if case["keep"] else {"y": y}
    if case["accumulate"]:
        block.copy_(s["other"])  # the other use's gradient arrives first
    dx = sim.gated_ff_grad(s["dy"], s["x"], s["hidden"], *columns, act=case["act"], accumulate=case["accumulate"])
    return {"dx": dx, "grads": block}


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    n = case["n"]
    if case["op"] == "orth":
        small, wide = sorted((case["rows"], case["cols"]))
        c = n * case["count"]
        # X X^T and its square are symmetric: half of each has to be computed
        return {"bytes": c * small * wide * (16 if case["velocity"] else 8),
                "flops": 5 * c * (small * small * wide + small ** 3 + 2 * small * small * wide)}
    size = 4 if case["dtype"] == "f32" else 2
    T, D, F = case["T"], case["D"], case["F"]
    cells, weights = n * T, 12 * n * D * F
    if case["op"] == "ff":
        return {"bytes": weights + size * cells * (2 * D + (2 * F if case["keep"] else 0)), "flops": 6 * cells * D * F}
    return {"bytes": weights * (3 if case["accumulate"] else 2) + size * cells * (3 * D + 2 * F), "flops": 12 * cells * D * F}


# ---- the definitions in 64 bits, apart from the plain form -----------------------------------------------------------------

def _exact_orth(case, s):
    count, rows, cols = case["count"], case["rows"], case["cols"]
    g = s["grad"].double()
    v = None if s["v"] is None else _MU * s["v"].double() + g
    u = g if v is None else g + _MU * v if case["nesterov"] else v
    updates = []
    for m in u.reshape(-1, rows, cols):
        x = m / (torch.linalg.norm(m) + _EPS)
        for _ in range(5):
            if rows <= cols:
                a = x @ x.T
                x = _P * x + _Q * (a @ x) + _R * (a @ (a @ x))
            else:
                a = x.T @ x
                x = _P * x + _Q * (x @ a) + _R * ((x @ a) @ a)
        updates.append(math.sqrt(max(1.0, rows / cols)) * x)
    out = {"update": torch.stack(updates).reshape(case["n"], count * rows * cols)}
    return out if v is None else dict(out, v=v)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "orth":
        return _exact_orth(case, s)
    n, D, F, off = case["n"], case["D"], case["F"], case["off"]
    ys, hs, dxs, gs = [], [], [], []
    for i in range(n):
        w = s["X"][i, off:].double()
        wg, wu, wd = w[:F * D].view(F, D), w[F * D:2 * F * D].view(F, D), w[2 * F * D:].view(D, F)
        x = s["x"][i].double()
        if case["op"] == "ff":
            a, b = x @ wg.T, x @ wu.T
            h = (a * torch.sigmoid(a) if case["act"] == "silu" else a * torch.special.ndtr(a)) * b
            ys.append(h @ wd.T)
            if case["keep"]:
                hs.append(torch.cat([a, b], dim=1))
            continue
        dy = s["dy"][i].double()
        a, b = s["hidden"][i, :, :F].double(), s["hidden"][i, :, F:].double()
        if case["act"] == "silu":
            q = torch.sigmoid(a)
            value, slope = a * q, q + a * q * torch.sigmoid(-a)
        else:
            q = torch.special.ndtr(a)
            value, slope = a * q, q + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
        dh = dy @ wd
        da, db = dh * b * slope, dh * value
        dxs.append(da @ wg + db @ wu)
        grads = torch.cat([(da.T @ x).reshape(-1), (db.T @ x).reshape(-1), (dy.T @ (value * b)).reshape(-1)])
        gs.append(grads + s["other"][i].double() if case["accumulate"] else grads)
    if case["op"] == "ff":
        return {"y": torch.stack(ys), "hidden": torch.stack(hs)} if case["keep"] else {"y": torch.stack(ys)}
    return {"dx": torch.stack(dxs), "grads": torch.stack(gs)}
