"""Training operators of the dense layers, each in a plain form and through the package.

Dense layers with bias, activation and residual (forward and backward), the same with one
weight per group of rows (node types, categories), the Newton-Schulz orthogonalisation of an
update and the optimiser step made of it. Each case is a dict of plain values; `listed()` gives
the fixed ones and `draw(rng)` another of the same ranges. `prepare` makes what a program holds
before the call, `run` is one pass through one operator, `exact` is its definition in 64 bits.

With `own` false, `run` computes the plain form in elementary torch operations in 32 bits,
rounded once at the end; with `own` true it calls the package.
"""

import math

import torch

own = False

DEV = "cuda"
COEFF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
BETA, LR, DECAY = 0.95, 0.02, 0.01
ACTIVATIONS = ("none", "relu", "gelu", "silu")


# ---- the cases -----------------------------------------------------------------------------
def listed():
    return [
        # One query's embedding through a wide output layer while it is served: latency.
        _dense("dense_fwd_query_bf16", "dense_fwd", 1, 1024, 2048, "bf16", "relu"),
        # The targets of a training minibatch (2,048 pairs and 500 negatives) through a hidden
        # layer with a residual, keeping what the backward pass needs; fp32.
        _dense("dense_fwd_batch_f32", "dense_fwd", 4596, 512, 512, "f32", "gelu", residual=True,
               train=True),
        # All of 300,000 nodes through the wide transform: the largest product.
        _dense("dense_fwd_nodes_bf16", "dense_fwd", 300_000, 1024, 2048, "bf16", "relu"),
        # The gradients of a minibatch's hidden layer, bf16.
        _dense("dense_bwd_batch_bf16", "dense_bwd", 4596, 512, 256, "bf16", "silu"),
        # The gradients of a layer fitted to an odd number of nodes, fp32.
        _dense("dense_bwd_nodes_f32", "dense_bwd", 100_003, 256, 512, "f32", "gelu"),
        # A few rows of mixed categories at serving time: most groups have one row or none.
        _dense("grouped_fwd_few_bf16", "dense_fwd", 23, 512, 512, "bf16", "silu", groups=16,
               residual=True),
        # Pins and boards, each with its own weight, fp32.
        _dense("grouped_fwd_types_f32", "dense_fwd", 120_011, 256, 256, "f32", "relu", groups=2),
        # Many categories of uneven size, some empty: forward and backward of the same layer.
        _dense("grouped_fwd_many_bf16", "dense_fwd", 60_000, 1024, 512, "bf16", "gelu", groups=64,
               residual=True, train=True),
        _dense("grouped_bwd_many_bf16", "dense_bwd", 60_000, 1024, 512, "bf16", "gelu", groups=64),
        # The update of a small layer for each of 8 groups, and of one wide fp32 layer.
        dict(name="orthogonalize_groups_bf16", kind="orthogonalize", batch=8, rows=256, cols=512,
             dtype="bf16"),
        dict(name="orthogonalize_wide_f32", kind="orthogonalize", batch=1, rows=2048, cols=1024,
             dtype="f32"),
        # The optimiser's whole step on the wide transform's weight.
        dict(name="muon_step_wide_bf16", kind="muon_step", batch=1, rows=2048, cols=2048,
             dtype="bf16"),
    ]


def draw(rng):
    kind = rng.choice(["dense_fwd", "dense_fwd", "dense_bwd", "grouped_fwd", "grouped_bwd",
                       "orthogonalize", "muon_step"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("orthogonalize", "muon_step"):
        # The larger of the two sides stays below 2048, the work below the largest listed one's.
        rows, cols = _side(rng, 16, 2048), _side(rng, 16, 2048)
        short, long = min(rows, cols), max(rows, cols)
        most = 2048 ** 2 * 1024 // (short * short * long)
        return dict(kind=kind, batch=_log(rng, 1, max(1, min(8, most))), rows=rows, cols=cols,
                    dtype=dtype)
    grouped = kind.startswith("grouped")
    d_in, d_out = _side(rng, 16, 2048), _side(rng, 16, 2048)
    groups = _log(rng, 2, 64) if grouped else 0
    cost = 60_000 * 1024 * 512 if grouped or kind == "dense_bwd" else 300_000 * 1024 * 2048
    if dtype == "f32":
        cost = min(cost, 100_003 * 256 * 512)
    rows = _log(rng, 1, max(2, min(300_000, cost // (d_in * d_out))))
    c = _dense("", "dense_" + kind.split("_")[1], rows, d_in, d_out, dtype,
               rng.choice(ACTIVATIONS), groups=groups, residual=rng.random() < 0.5,
               train=rng.random() < 0.5)
    c.pop("name")
    return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, lo, hi):
    """A layer's width: half of them multiples of 16, the others anything."""
    v = _log(rng, lo, hi)
    return max(lo, v // 16 * 16) if rng.random() < 0.5 else v


def _dense(name, kind, rows, d_in, d_out, dtype, act, groups=0, residual=False, train=False):
    back = kind == "dense_bwd"
    return dict(name=name, kind=kind, rows=rows, d_in=d_in, d_out=d_out, dtype=dtype, act=act,
                groups=groups, residual=residual and not back, train=train and not back)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- what a program holds before the call --------------------------------------------------
def _group_sizes(rows, groups, gen):
    """Uneven group sizes that add up to `rows`: Zipf-like over a random order, with more than
    two groups every fifth one empty."""
    share = [1.0 / (i + 1) ** 0.8 for i in range(groups)]
    if groups > 2:
        share = [0.0 if i % 5 == 4 else s for i, s in enumerate(share)]
    total = sum(share)
    sizes = [int(rows * s / total) for s in share]
    for i in range(rows - sum(sizes)):
        sizes[i % groups if share[i % groups] else 0] += 1
    order = torch.randperm(groups, generator=gen).tolist()
    return [sizes[i] for i in order]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device=DEV) * scale

    if case["kind"] in ("orthogonalize", "muon_step"):
        b, m, n = case["batch"], case["rows"], case["cols"]
        # A gradient: a few strong directions over noise, of the size that a mean loss gives.
        k = max(1, min(m, n) // 16)
        g = normal(b, m, k) @ normal(b, k, n) / math.sqrt(k) + normal(b, m, n, scale=0.5)
        s = dict(case=case, g=(g * 1e-3).to(dt))
        if case["kind"] == "muon_step":
            lim = math.sqrt(6.0 / (m + n))
            s["W"] = ((torch.rand(b, m, n, generator=gen, device=DEV) * 2 - 1) * lim).to(dt)
            s["momentum"] = normal(b, m, n, scale=5e-3)
            s["W_new"], s["momentum_new"] = torch.empty_like(s["W"]), torch.empty_like(s["momentum"])
        return s

    n, d_in, d_out, groups = case["rows"], case["d_in"], case["d_out"], case["groups"]
    lead = (groups,) if groups else ()
    lim = math.sqrt(6.0 / (d_in + d_out))
    s = dict(case=case, x=normal(n, d_in).to(dt),
             W=((torch.rand(*lead, d_out, d_in, generator=gen, device=DEV) * 2 - 1) * lim).to(dt),
             b=(torch.rand(*lead, d_out, generator=gen, device=DEV) * 2 - 1) * 0.1,
             offsets=None, bounds=[(0, n)], residual=None)
    if groups:
        ends = [0]
        for v in _group_sizes(n, groups, host):
            ends.append(ends[-1] + v)
        s["bounds"] = list(zip(ends[:-1], ends[1:]))
        s["offsets"] = torch.tensor(ends, dtype=torch.int64, device=DEV)
    if case["residual"]:
        s["residual"] = normal(n, d_out).to(dt)
    if case["kind"] == "dense_bwd":
        s["dy"] = normal(n, d_out, scale=1.0 / n).to(dt)
        # The pre-activation that the forward pass kept.
        s["u"] = _pre_activation(s).to(dt)
    return s


# ---- the plain forms, in 32 bits -----------------------------------------------------------
def _pre_activation(s):
    x, W = s["x"].float(), s["W"].float()
    if s["offsets"] is None:
        return x @ W.t() + s["b"]
    u = x.new_empty(x.shape[0], W.shape[1])
    for g, (lo, hi) in enumerate(s["bounds"]):
        u[lo:hi] = x[lo:hi] @ W[g].t() + s["b"][g]
    return u


def _activate(u, act):
    if act == "relu":
        return torch.where(u > 0, u, torch.zeros_like(u))
    if act == "gelu":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u)))
    if act == "silu":
        return u / (1 + torch.exp(-u))
    return u


def _slope(u, act):
    """The activation's derivative."""
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u))
        return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * math.sqrt(2 / math.pi) * (
            1 + 3 * 0.044715 * u * u)
    if act == "silu":
        p = 1 / (1 + torch.exp(-u))
        return p * (1 + u * (1 - p))
    return torch.ones_like(u)


def _plain_forward(s):
    c, dt = s["case"], s["x"].dtype
    u = _pre_activation(s)
    y = _activate(u, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(dt), u.to(dt)) if c["train"] else y.to(dt)


def _plain_backward(s):
    c, dt = s["case"], s["x"].dtype
    x, W = s["x"].float(), s["W"].float()
    dz = s["dy"].float() * _slope(s["u"].float(), c["act"])
    if s["offsets"] is None:
        return (dz @ W).to(dt), (dz.t() @ x).to(dt), dz.sum(0)
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(s["b"])
    for g, (lo, hi) in enumerate(s["bounds"]):
        dx[lo:hi] = dz[lo:hi] @ W[g]
        dW[g] = dz[lo:hi].t() @ x[lo:hi]
        db[g] = dz[lo:hi].sum(0)
    return dx.to(dt), dW.to(dt), db


def _newton_schulz(g):
    a, b, c = COEFF
    tall = g.shape[-2] > g.shape[-1]
    X = g.transpose(-1, -2).contiguous() if tall else g
    X = X / (torch.sqrt((X * X).sum((-2, -1), keepdim=True)) + EPS)
    for _ in range(5):
        A = X @ X.transpose(-1, -2).contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.transpose(-1, -2).contiguous() if tall else X


def _scale(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def _plain_muon(s):
    g = s["g"].float()
    momentum = BETA * s["momentum"] + g
    O = _newton_schulz(g + BETA * momentum)
    W = (1 - LR * DECAY) * s["W"].float() - LR * _scale(s["case"]) * O
    return W.to(s["W"].dtype), momentum


# ---- one pass ------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if not own:
        if case["kind"] == "dense_fwd":
            return _plain_forward(state)
        if case["kind"] == "dense_bwd":
            return _plain_backward(state)
        if case["kind"] == "orthogonalize":
            return _newton_schulz(state["g"].float()).to(state["g"].dtype)
        return _plain_muon(state)

    import paper_1806_01973_amd as ps
    if case["kind"] == "dense_fwd":
        return ps.dense_forward(state["x"], state["W"], state["b"], activation=case["act"],
                                residual=state["residual"], offsets=state["offsets"],
                                want_preact=case["train"])
    if case["kind"] == "dense_bwd":
        return ps.dense_backward(state["dy"], state["x"], state["W"], state["u"],
                                 activation=case["act"], offsets=state["offsets"])
    if case["kind"] == "orthogonalize":
        return ps.orthogonalize(state["g"])
    return ps.muon_step(state["W"], state["g"], state["momentum"], lr=LR, beta=BETA,
                        weight_decay=DECAY, W_out=state["W_new"],
                        momentum_out=state["momentum_new"])


# ---- what a pass cannot do without ---------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("orthogonalize", "muon_step"):
        size = case["batch"] * case["rows"] * case["cols"]
        m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # A and A A are symmetric: half of each product.
        flops = 5 * case["batch"] * (3 * m * m * n + m * m * m)
        if case["kind"] == "orthogonalize":
            return {"bytes": 2 * size * es, "flops": flops}
        return {"bytes": size * (3 * es + 8), "flops": flops}
    n, d_in, d_out, groups = case["rows"], case["d_in"], case["d_out"], max(1, case["groups"])
    x, y, w = n * d_in * es, n * d_out * es, groups * d_in * d_out * es
    bias = groups * d_out * 4
    if case["kind"] == "dense_fwd":
        return {"bytes": x + w + bias + y * (1 + case["residual"] + case["train"]),
                "flops": 2 * n * d_in * d_out}
    return {"bytes": 2 * (x + w + y) + bias, "flops": 4 * n * d_in * d_out}


# ---- the definitions in 64 bits ------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    if case["kind"] in ("orthogonalize", "muon_step"):
        u = s["g"].to(D)
        if case["kind"] == "muon_step":
            momentum = s["momentum"].to(D) * BETA + u
            u = u + momentum * BETA
        out = []
        for M in u:
            flip = M.shape[0] > M.shape[1]
            Y = (M.t() if flip else M).contiguous()
            Y = Y / (torch.linalg.vector_norm(Y) + EPS)
            for _ in range(5):
                S = torch.mm(Y, Y.t().contiguous())
                # a I + b S + c S^2 applied from the left
                P = COEFF[1] * S + COEFF[2] * torch.mm(S, S)
                P.diagonal().add_(COEFF[0])
                Y = torch.mm(P, Y)
            out.append(Y.t().contiguous() if flip else Y)
        O = torch.stack(out)
        if case["kind"] == "orthogonalize":
            return O
        return s["W"].to(D) * (1 - LR * DECAY) - O * (LR * _scale(case)), momentum

    groups = case["groups"]
    W = s["W"].to(D).reshape(max(1, groups), case["d_out"], case["d_in"])
    b = s["b"].to(D).reshape(max(1, groups), case["d_out"])
    if case["kind"] == "dense_fwd":
        u = torch.cat([torch.addmm(b[g], s["x"][lo:hi].to(D), W[g].t().contiguous())
                       for g, (lo, hi) in enumerate(s["bounds"])])
        y = {"none": lambda v: v, "relu": torch.relu,
             "gelu": lambda v: torch.nn.functional.gelu(v, approximate="tanh"),
             "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](u)
        if s["residual"] is not None:
            y = y + s["residual"].to(D)
        return (y, u) if case["train"] else y
    u = s["u"].to(D)
    if case["act"] == "relu":
        slope = torch.where(u > 0, 1.0, 0.0)
    elif case["act"] == "gelu":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * u * (1 + 0.044715 * u.square()))
        slope = (1 + t) / 2 + u / 2 * (1 - t.square()) * k * (1 + 0.134145 * u.square())
    elif case["act"] == "silu":
        t = torch.sigmoid(u)
        slope = t + u * t * (1 - t)
    else:
        slope = torch.ones_like(u)
    dz = s["dy"].to(D) * slope
    dx, dW, db = [], [], []
    for g, (lo, hi) in enumerate(s["bounds"]):
        part = dz[lo:hi]
        dx.append(torch.mm(part, W[g]))
        dW.append(torch.mm(part.t().contiguous(), s["x"][lo:hi].to(D)))
        db.append(part.sum(0))
    dx, dW, db = torch.cat(dx), torch.stack(dW), torch.stack(db)
    return (dx, dW, db) if groups else (dx, dW[0], db[0])
