"""Performance cases of the language-model operators: what stands between the tokens of n nodes and the gradients in G.

Every node i has parameters of its own, a row of X; the operators read them there, at a column offset, and write their
gradients to the same columns of G.  Activations are (n, T, D) tensors, T tokens a node.

  embed       y[i,t] = scale * E_i[token[i,t]]; a token below 0 is padding and gives a row of zeros
  embed_grad  dE_i[v] = scale * sum of dy[i,t] over the t with token v, into G (or added to what is there)
  dropout     y = residual + mask * x / (1 - p), the mask from Philox4x32-10 addressed by (seed, layer, node, iteration, t, c)
  norm        u = residual + dropout(x); y = gamma_i * (u - mean) / sqrt(var + eps) + beta_i
  norm_grad   gradients with respect to u and x, and those of gamma_i and beta_i, summed over the tokens, into G
  loss        cross-entropy of softmax(z) against the label, averaged over a node's tokens with a label >= 0, and its
              gradient with respect to z

Where `own` is false the same results come from elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5


def listed():
    return [
        # One new token a node looked up in a vocabulary of 32000 rows of 768 floats: a model answering token by token.  Latency.
        dict(name="embed_next_token", op="embed", n=8, T=1, V=32000, D=768, dtype="f32", off=0),
        # The input of a training step: 8 sequences of 512 tokens on each of 8 nodes, frequent tokens often, a tail of padding.
        dict(name="embed_batch", op="embed", n=8, T=4096, V=32000, D=768, dtype="bf16", off=0),
        # The gradient of that table: G is written whole, rows of tokens that did not occur with zeros.
        dict(name="embed_grad_batch", op="embed_grad", n=8, T=4096, V=32000, D=768, dtype="bf16", off=0, accumulate=False),
        # A small vocabulary whose table is also the output layer: its gradient is added to that layer's.  Odd everywhere.
        dict(name="embed_grad_tied_odd", op="embed_grad", n=5, T=4099, V=1013, D=257, dtype="f32", off=7, accumulate=True),
        # Layer norm of one new token a node, as in evaluation: no residual, no dropout.  Latency.
        dict(name="norm_next_token", op="norm", n=8, T=1, D=768, dtype="f32", off=0, p=0.0, residual=False),
        # Dropout, residual sum and layer norm of a training step in bf16.
        dict(name="norm_batch", op="norm", n=8, T=4096, D=768, dtype="bf16", off=0, p=0.1, residual=True),
        # Its backward pass, with the sums over tokens that make the gradients of gamma and beta.
        dict(name="norm_grad_batch", op="norm_grad", n=8, T=4096, D=768, dtype="bf16", off=0, p=0.1, more=False),
        # Rows that no vector width divides, in half precision; u goes on as the residual stream, whose gradient is added.
        dict(name="norm_grad_odd", op="norm_grad", n=7, T=1021, D=1023, dtype="f16", off=5, p=0.0, more=True),
        # A short ragged batch on twenty nodes.
        dict(name="dropout_small_odd", op="dropout", n=20, T=33, D=129, dtype="f32", p=0.5, residual=False),
        # The sum of a sublayer's output and the residual stream on sixteen nodes: bytes and generator together.
        dict(name="dropout_wide", op="dropout", n=16, T=8192, D=1024, dtype="bf16", p=0.1, residual=True),
        # Next-token loss and its gradient over the whole vocabulary, a tail of padding.
        dict(name="loss_batch", op="loss", n=8, T=512, V=32000, dtype="bf16", grad=True, counted=0.9),
        # The loss of one token a node over a large vocabulary, without a gradient: few long rows.
        dict(name="loss_one_token", op="loss", n=4, T=1, V=128000, dtype="f32", grad=False, counted=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' range; no array is larger than the largest of the listed ones (786 MB of G)."""
    op = rng.choice(["embed", "embed_grad", "embed_grad", "dropout", "norm", "norm_grad", "norm_grad", "loss", "loss"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    n = _log_int(rng, 1, 32)
    T = _log_int(rng, 1, 8192)
    if op in ("embed", "embed_grad"):
        D = _log_int(rng, 16, 4096)
        V = _log_int(rng, 32, 128000)
        V = max(2, min(V, 150_000_000 // (n * D)))
        T = max(1, min(T, 100_000_000 // (n * D)))
        c = dict(op=op, n=n, T=T, V=V, D=D, dtype=dtype, off=rng.choice([0, 0, 1, 2 * D, 13]))
        return dict(c, accumulate=rng.random() < 0.4) if op == "embed_grad" else c
    if op == "loss":
        V = _log_int(rng, 32, 128000)
        T = max(1, min(T, 100_000_000 // (n * V)))
        return dict(op=op, n=n, T=T, V=V, dtype=dtype, grad=rng.random() < 0.75, counted=rng.choice([1.0, 0.9, 0.15]))
    D = _log_int(rng, 16, 8192)
    T = max(1, min(T, 60_000_000 // (n * D)))
    p = rng.choice([0.0, 0.1, 0.1, 0.25, 0.5])
    if op == "dropout":
        return dict(op=op, n=n, T=T, D=D, dtype=dtype, p=p or 0.1, residual=rng.random() < 0.5)
    c = dict(op=op, n=n, T=T, D=D, dtype=dtype, off=rng.choice([0, 0, 1, D, 11]), p=p)
    return dict(c, residual=rng.random() < 0.6) if op == "norm" else dict(c, more=rng.random() < 0.4)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _columns(case):
    """Parameters a node has: a block of `off` floats that belongs to other layers, then this one's."""
    if case["op"] in ("embed", "embed_grad"):
        return case["off"] + case["V"] * case["D"]
    if case["op"] in ("norm", "norm_grad"):
        return case["off"] + 2 * case["D"]
    return 4


def _tokens(case, g):
    """Token frequencies fall as 1 / rank (a log-uniform draw); the last tenth of longer sequences is padding (-1)."""
    n, T, V = case["n"], case["T"], case["V"]
    u = torch.rand((n, T), device="cuda", generator=g, dtype=torch.float64)
    tok = (torch.exp(u * math.log(V + 1.0)).floor() - 1).clamp_(0, V - 1).to(torch.int32)
    if T >= 10:
        tok[:, T - T // 10:] = -1
    return tok


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, n, d = case["op"], case["n"], _columns(case)
    dtype = _DTYPE[case["dtype"]]
    s = dict(case=case, seed=(seed * 0x9E3779B97F4A7C15 + 1) & 0xFFFFFFFFFFFFFFFF, layer=seed % 97)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=g) * scale

    X = normal(n, d, scale=0.02)
    if op in ("norm", "norm_grad"):
        X[:, case["off"]:case["off"] + case["D"]] += 1.0
    if op in ("embed", "embed_grad"):
        s["tokens"] = _tokens(case, g)
        s["scale"] = math.sqrt(case["D"])
    if op == "embed_grad":
        s["dy"] = normal(n, case["T"], case["D"], scale=1e-2).to(dtype)
        if case["accumulate"]:
            s["other"] = normal(n, case["V"] * case["D"], scale=1e-2)
    if op in ("dropout", "norm"):
        s["x"] = normal(n, case["T"], case["D"]).to(dtype)
        s["residual"] = (normal(n, case["T"], case["D"]) + 0.25).to(dtype) if case["residual"] else None
    if op == "norm_grad":
        s["dy"] = normal(n, case["T"], case["D"], scale=1e-2).to(dtype)
        s["u"] = (normal(n, case["T"], case["D"], scale=1.4) + 0.25).to(dtype)
        u = s["u"].float()
        mean = u.mean(dim=2)
        s["stats"] = torch.stack([mean, ((u - mean[..., None]).square().mean(dim=2) + _EPS).rsqrt()], dim=2).contiguous()
        s["more"] = normal(n, case["T"], case["D"], scale=1e-2).to(dtype) if case["more"] else None
    if op == "loss":
        n, T, V = n, case["T"], case["V"]
        s["logits"] = normal(n, T, V, scale=2.0).to(dtype)
        label = torch.randint(0, V, (n, T), device="cuda", generator=g, dtype=torch.int32)
        dropped = torch.rand((n, T), device="cuda", generator=g) >= case["counted"]
        s["labels"] = torch.where(dropped, torch.full_like(label, -1), label)
        s["grad_scale"] = 1024.0 if case["dtype"] == "f16" else 1.0
    if own:
        from paper_2105_09080_amd.harness import Simulation
        s["sim"] = Simulation(n, d, topology="ring", H=6, lr=0.1)
        s["sim"].X.copy_(X)
    else:
        s["X"] = X
    return s


# ---- the operators in their plain form ----------------------------------------------------------------------------------

def _mask(s, T, D):
    """Dropout's mask and factor.  Counter words (8 columns of a row, node, iteration 0, 4 + 256 * layer), the key is the
    seed; each of the four 32-bit words holds two lots of 16 bits, the lower half first; an element stays if its lot is
    at least 65536 p."""
    n, p = s["case"]["n"], s["case"]["p"]
    low = 0xFFFFFFFF
    groups = (D + 7) // 8
    c0 = torch.arange(T * groups, device="cuda", dtype=torch.int64).view(1, -1).expand(n, -1)
    c1 = torch.arange(n, device="cuda", dtype=torch.int64).view(-1, 1)
    c2 = torch.zeros_like(c1)
    c3 = torch.full_like(c1, 4 + 256 * s["layer"])
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for r in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([w.expand(n, T * groups) for w in (c0, c1, c2, c3)], dim=2)
    lots = torch.stack([words & 0xFFFF, words >> 16], dim=3).view(n, T, groups * 8)[:, :, :D]
    drop = int(p * 65536 + 0.5)
    return lots >= drop, 65536.0 / (65536 - drop)


def _dropped(s, x):
    """mask * x / (1 - p) in 32 bits."""
    if s["case"]["p"] == 0.0:
        return x
    keep, factor = _mask(s, x.shape[1], x.shape[2])
    return torch.where(keep, x * factor, torch.zeros((), device="cuda"))


def _gamma_beta(s):
    off, D = s["case"]["off"], s["case"]["D"]
    return s["X"][:, None, off:off + D], s["X"][:, None, off + D:off + 2 * D]


def _plain(s):
    case = s["case"]
    op, n = case["op"], case["n"]
    dtype = _DTYPE[case["dtype"]]
    if op == "embed":
        V, D = case["V"], case["D"]
        table = s["X"][:, case["off"]:].reshape(n, V, D)
        tok = s["tokens"].long()
        rows = table[torch.arange(n, device="cuda")[:, None], tok.clamp(min=0)] * s["scale"]
        return torch.where((tok >= 0)[..., None], rows, torch.zeros((), device="cuda")).to(dtype)
    if op == "embed_grad":
        V, D = case["V"], case["D"]
        tok = s["tokens"].long()
        at = torch.where(tok >= 0, tok, V) + torch.arange(n, device="cuda")[:, None] * (V + 1)
        sums = torch.zeros((n * (V + 1), D), device="cuda").index_add_(0, at.view(-1), s["dy"].float().view(-1, D) * s["scale"])
        table = sums.view(n, V + 1, D)[:, :V].reshape(n, V * D)
        return s["other"] + table if case["accumulate"] else table
    if op == "dropout":
        y = _dropped(s, s["x"].float())
        return (y if s["residual"] is None else y + s["residual"].float()).to(dtype)
    if op == "norm":
        u = _dropped(s, s["x"].float())
        u = u if s["residual"] is None else u + s["residual"].float()
        mean = u.mean(dim=2, keepdim=True)
        rstd = ((u - mean).square().mean(dim=2, keepdim=True) + _EPS).rsqrt()
        gamma, beta = _gamma_beta(s)
        y = ((u - mean) * rstd * gamma + beta).to(dtype)
        return {"y": y, "u": u.to(dtype), "stats": torch.cat([mean, rstd], dim=2)}
    if op == "norm_grad":
        mean, rstd = s["stats"][..., :1], s["stats"][..., 1:]
        dy = s["dy"].float()
        xh = (s["u"].float() - mean) * rstd
        h = dy * _gamma_beta(s)[0]
        du = rstd * (h - h.mean(dim=2, keepdim=True) - xh * (h * xh).mean(dim=2, keepdim=True))
        du = du if s["more"] is None else du + s["more"].float()
        return {"du": du.to(dtype), "dx": _dropped(s, du).to(dtype), "dgamma": (dy * xh).sum(dim=1), "dbeta": dy.sum(dim=1)}
    z = s["logits"].float()
    label = s["labels"].long()
    counted = label >= 0
    top = z.amax(dim=2, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=2, keepdim=True)
    at = label.clamp(min=0)[..., None]
    rows = torch.log(total[..., 0]) + top[..., 0] - z.gather(2, at)[..., 0]
    count = counted.sum(dim=1).clamp(min=1).float()
    out = {"loss": torch.where(counted, rows, torch.zeros((), device="cuda")).sum(dim=1) / count}
    if case["grad"]:
        grad = e / total
        grad.scatter_add_(2, at, torch.full_like(at, -1, dtype=torch.float32))
        grad *= torch.where(counted, (s["grad_scale"] / count)[:, None], torch.zeros((), device="cuda"))[..., None]
        out["dlogits"] = grad.to(dtype)
    return out


# ---- the framework's calls ------------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    case, sim = s["case"], s["sim"]
    op = case["op"]
    dtype = _DTYPE[case["dtype"]]
    if op == "embed":
        return sim.embed(s["tokens"], case["off"], case["V"], case["D"], scale=s["scale"], dtype=dtype)
    if op == "embed_grad":
        block = sim.G[:, case["off"]:]
        if case["accumulate"]:
            block.copy_(s["other"])  # the output layer's gradient arrives first
        sim.embed_grad(s["tokens"], s["dy"], case["off"], case["V"], scale=s["scale"], accumulate=case["accumulate"])
        return block
    if op == "dropout":
        return sim.dropout(s["x"], case["p"], seed=s["seed"], layer=s["layer"], residual=s["residual"])
    if op == "norm":
        off, D = case["off"], case["D"]
        y, u, stats = sim.layer_norm(s["x"], off, off + D, eps=_EPS, residual=s["residual"], p=case["p"], seed=s["seed"],
                                     layer=s["layer"])
        return {"y": y, "u": u, "stats": stats}
    if op == "norm_grad":
        off, D = case["off"], case["D"]
        du, dx = sim.layer_norm_grad(s["dy"], s["u"], s["stats"], off, off + D, p=case["p"], seed=s["seed"],
                                     layer=s["layer"], more=s["more"])
        return {"du": du, "dx": dx, "dgamma": sim.G[:, off:off + D], "dbeta": sim.G[:, off + D:off + 2 * D]}
    loss, dlogits = sim.token_loss(s["logits"], s["labels"], grad=case["grad"], grad_scale=s["grad_scale"])
    return {"loss": loss, "dlogits": dlogits} if case["grad"] else {"loss": loss}


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def _distinct(case):
    """Expected distinct tokens of a node: V tokens drawn with probability log((r+2)/(r+1)) / log(V+1)."""
    T, V = case["T"] - (case["T"] // 10 if case["T"] >= 10 else 0), case["V"]
    r = torch.arange(V, dtype=torch.float64)
    p = torch.log((r + 2) / (r + 1)) / math.log(V + 1.0)
    return float((1 - (1 - p) ** T).sum())


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    op, n, T = case["op"], case["n"], case["T"]
    if op == "loss":
        rows, V = n * T, case["V"]
        counted = rows * case["counted"]
        return {"bytes": 4 * rows + 4 * n + size * counted * V + (size * rows * V if case["grad"] else 0), "flops": 4 * counted * V}
    D = case["D"]
    cells = n * T * D
    if op == "embed":
        return {"bytes": 4 * n * T + 4 * n * D * _distinct(case) + size * cells, "flops": cells}
    if op == "embed_grad":
        kept = T - (T // 10 if T >= 10 else 0)
        g = 4 * n * case["V"] * D * (2 if case["accumulate"] else 1)  # the other gradient is read, the sum written
        return {"bytes": 4 * n * T + size * n * kept * D + g, "flops": n * kept * D}
    if op == "dropout":
        return {"bytes": size * cells * (3 if case["residual"] else 2), "flops": 2 * cells}
    if op == "norm":
        arrays = 2 + (1 if case["residual"] else 0) + (1 if case["residual"] or case["p"] else 0)
        return {"bytes": size * cells * arrays + 8 * n * T + 8 * n * D, "flops": 8 * cells}
    arrays = 3 + (1 if case["more"] else 0) + (1 if case["p"] else 0)
    return {"bytes": size * cells * arrays + 8 * n * T + 12 * n * D, "flops": 14 * cells}


# ---- the definitions in 64 bits, apart from the plain form -----------------------------------------------------------------

def _exact_dropped(s, x):
    """As the definition has it, element by element, with products of 16-bit pieces in place of 64-bit ones."""
    p = s["case"]["p"]
    if p == 0.0:
        return x
    n, T, D = x.shape
    m16 = 0xFFFF

    def product(a, m):
        al, ah, ml, mh = a & m16, a >> 16, m & m16, m >> 16
        ll, lh, hl, hh = al * ml, al * mh, ah * ml, ah * mh
        mid = (ll >> 16) + (lh & m16) + (hl & m16)
        return hh + (lh >> 16) + (hl >> 16) + (mid >> 16), ((mid & m16) << 16) | (ll & m16)

    row = torch.arange(T, device="cuda", dtype=torch.int64)[:, None] * ((D + 7) // 8)
    w = [(row + torch.arange((D + 7) // 8, device="cuda", dtype=torch.int64)[None, :])[None].expand(n, -1, -1),
         torch.arange(n, device="cuda", dtype=torch.int64)[:, None, None], torch.zeros((1, 1, 1), device="cuda", dtype=torch.int64),
         torch.full((1, 1, 1), 4 + (s["layer"] << 8), device="cuda", dtype=torch.int64)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for _ in range(10):
        h0, l0 = product(w[0], 0xD2511F53)
        h1, l1 = product(w[2], 0xCD9E8D57)
        w = [h1 ^ w[1] ^ key[0], l1, h0 ^ w[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = torch.empty_like(x)
    lots = 65536 - int(p * 65536 + 0.5)
    for j in range(8):
        if j < D:
            lot = (w[j // 2] >> (16 * (j % 2))) & m16
            cols = x[:, :, j::8]
            out[:, :, j::8] = cols * (65536.0 / lots) * (lot[:, :, :cols.shape[2]] >= 65536 - lots).double()
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op, n = case["op"], case["n"]
    params = s["X"].double()
    if op in ("embed", "embed_grad"):
        V, D, off = case["V"], case["D"], case["off"]
        out = []
        for i in range(n):
            tok = s["tokens"][i].long()
            on = tok >= 0
            if op == "embed":
                y = torch.zeros((case["T"], D), device="cuda", dtype=torch.float64)
                y[on] = params[i, off:].view(V, D).index_select(0, tok[on]) * s["scale"]
            else:
                y = s["other"][i].double().view(V, D).clone() if case["accumulate"] else torch.zeros((V, D), device="cuda", dtype=torch.float64)
                y.index_put_((tok[on],), s["dy"][i][on].double() * s["scale"], accumulate=True)
                y = y.view(-1)
            out.append(y)
        return torch.stack(out)
    if op == "dropout":
        y = _exact_dropped(s, s["x"].double())
        return y if s["residual"] is None else y + s["residual"].double()
    if op in ("norm", "norm_grad"):
        off, D = case["off"], case["D"]
        gamma, beta = params[:, None, off:off + D], params[:, None, off + D:off + 2 * D]
    if op == "norm":
        u = _exact_dropped(s, s["x"].double()) + (0.0 if s["residual"] is None else s["residual"].double())
        var, mean = torch.var_mean(u, dim=2, keepdim=True, correction=0)
        sd = torch.sqrt(var + _EPS)
        return {"y": gamma * (u - mean) / sd + beta, "u": u, "stats": torch.cat([mean, 1.0 / sd], dim=2)}
    if op == "norm_grad":
        dy, more = s["dy"].double(), 0.0 if s["more"] is None else s["more"].double()
        mean, rstd = s["stats"].double().unbind(dim=2)
        xh = (s["u"].double() - mean[..., None]) * rstd[..., None]
        a = (gamma * dy).sum(dim=2) / D
        b = (gamma * dy * xh).sum(dim=2) / D
        du = rstd[..., None] * (gamma * dy - a[..., None] - b[..., None] * xh) + more
        return {"du": du, "dx": _exact_dropped(s, du), "dgamma": (dy * xh).sum(dim=1), "dbeta": dy.sum(dim=1)}
    z, label = s["logits"].double(), s["labels"].long()
    on = label >= 0
    logp = torch.log_softmax(z, dim=2)
    losses, grads = [], []
    for i in range(n):
        count = max(1, int(on[i].sum()))
        picked = logp[i, on[i], label[i, on[i]]]
        losses.append(-picked.sum() / count)
        if case["grad"]:
            g = torch.zeros_like(logp[i])
            g[on[i]] = logp[i, on[i]].exp()
            g[on[i], label[i, on[i]]] -= 1.0
            grads.append(g * (s["grad_scale"] / count))
    out = {"loss": torch.stack(losses)}
    if case["grad"]:
        out["dlogits"] = torch.stack(grads)
    return out
