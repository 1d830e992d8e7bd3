"""The operators a model needs next to the minibatches that this package prepares: what is measured of them.

A batch arrives as feature rows (`out_rows` of a cache lookup: fp32 or bf16, each row padded to 16 bytes) and node ids.
  linear       one layer over the rows: product, bias, residual and activation; with its gradients where `train` is set
  grouped      the same with a weight per node type: the ids are sorted by type, each type's rows meet its own matrix
  orthogonal   a weight gradient made (nearly) orthogonal by five Newton-Schulz steps before it is applied

The plain forms below are elementary torch operations in 32 bits; `exact` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def listed():
    return [
        # One node's prediction: a single row through a wide layer, where the call itself is the cost.
        dict(name="linear one row", kind="linear", dtype="bf16", rows=1, in_dim=512, out_dim=512,
             activation="relu", residual="none", bias=True, train=False),
        # The input layer over a small batch (a test or a small dataset), fp32 rows of 100 values.
        dict(name="linear small", kind="linear", dtype="f32", rows=5_485, in_dim=100, out_dim=128,
             activation="relu", residual="none", bias=True, train=False),
        # A training step of the input layer over an ordinary batch: forward, then all three gradients, fp32.
        dict(name="linear train f32", kind="linear", dtype="f32", rows=428_377, in_dim=100, out_dim=256,
             activation="gelu", residual="none", bias=True, train=True),
        # The same over the wide bf16 rows; the neighbours' share joins before the activation.
        dict(name="linear train bf16", kind="linear", dtype="bf16", rows=302_709, in_dim=512, out_dim=256,
             activation="relu", residual="before", bias=True, train=True),
        # A residual layer as wide as the rows, forward only: the largest batch of an evaluation.
        dict(name="linear wide", kind="linear", dtype="bf16", rows=302_709, in_dim=512, out_dim=512,
             activation="silu", residual="after", bias=True, train=False),
        # A few nodes of several types answered at once.
        dict(name="grouped few rows", kind="grouped", dtype="bf16", rows=37, in_dim=256, out_dim=256, groups=8, empty=2,
             left_out=0.0, activation="none", residual="none", bias=True, train=False),
        # A training step of the typed input layer over a small batch; some nodes have no type.
        dict(name="grouped small train", kind="grouped", dtype="f32", rows=5_485, in_dim=100, out_dim=64, groups=4, empty=0,
             left_out=0.02, activation="silu", residual="none", bias=True, train=True),
        # The typed input layer over an ordinary batch, fp32, forward only.
        dict(name="grouped f32", kind="grouped", dtype="f32", rows=428_377, in_dim=100, out_dim=128, groups=8, empty=1,
             left_out=0.0, activation="relu", residual="none", bias=True, train=False),
        # A training step of the typed input layer over wide bf16 rows, many types of very different sizes.
        dict(name="grouped train bf16", kind="grouped", dtype="bf16", rows=302_709, in_dim=512, out_dim=256, groups=24, empty=3,
             left_out=0.0, activation="gelu", residual="none", bias=True, train=True),
        # The update of a small layer for each of a few types: launches and latency count.
        dict(name="orthogonal small", kind="orthogonal", dtype="f32", batch=4, rows=128, cols=100, steps=5),
        # The update of the typed input layer: one matrix for each type, bf16.
        dict(name="orthogonal types", kind="orthogonal", dtype="bf16", batch=24, rows=256, cols=512, steps=5),
        # The update of the widest layers, fp32.
        dict(name="orthogonal wide", kind="orthogonal", dtype="f32", batch=2, rows=2048, cols=1024, steps=5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "grouped", "grouped", "orthogonal"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "orthogonal":
        rows, cols = _log_int(rng, 24, 1280), _log_int(rng, 24, 1280)
        most = (1 << 31) // (min(rows, cols) ** 2 * max(rows, cols))
        return dict(kind=kind, dtype=dtype, batch=_log_int(rng, 1, max(1, min(24, most))), rows=rows, cols=cols, steps=5)
    train = rng.random() < 0.5
    in_dim, out_dim = _log_int(rng, 16, 640), _log_int(rng, 16, 512)
    # no more products, and no more memory, than the largest listed case of the type
    most = (10_000_000_000 if dtype == "f32" else 35_000_000_000) // (in_dim * out_dim)
    most = min(most, (150_000_000 if dtype == "f32" else 220_000_000) // (in_dim + out_dim), 428_377)
    rows = _log_int(rng, 1, most)
    # (in fp32 a relu's gradient jumps where two orders of summation give a product near zero different signs)
    activation = rng.choice(["none", "gelu", "silu"] if train and dtype == "f32" else ["none", "relu", "gelu", "silu"])
    case = dict(kind=kind, dtype=dtype, rows=rows, in_dim=in_dim, out_dim=out_dim, activation=activation,
                residual=rng.choice(["none", "none", "before", "after"]), bias=rng.random() < 0.75, train=train)
    if kind == "grouped":
        groups = _log_int(rng, 2, 48)
        case.update(groups=groups, empty=rng.randint(0, groups // 3), left_out=rng.choice([0.0, 0.0, 0.05]))
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 1)
    return g


def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def _layer(case, gen):
    """A layer's inputs: rows as a lookup leaves them (padded to 16 bytes), weights, and what comes back from above."""
    dtype = TYPES[case["dtype"]]
    n, k, m = case["rows"], case["in_dim"], case["out_dim"]
    g = case.get("groups", 1)
    lead = (g,) if case["kind"] == "grouped" else ()
    per = 16 // dtype.itemsize
    s = dict(case=case, dtype=dtype)
    s["x"] = _normal(gen, (n, -(-k // per) * per), dtype)[:, :k]
    s["weight"] = _normal(gen, lead + (m, k), dtype, 1.0 / math.sqrt(k))
    s["bias"] = _normal(gen, lead + (m,), dtype, 0.3) if case["bias"] else None
    s["residual"] = _normal(gen, (n, m), dtype, 0.7) if case["residual"] != "none" else None
    s["dy"] = _normal(gen, (n, m), dtype) if case["train"] else None
    return s


def _types(case, gen):
    """Ids of a batch and the type of every node: sizes fall like 1/(rank+1), the last `empty` types have no node."""
    n, g = case["rows"], case["groups"]
    nodes = 4 * n + 1000
    weight = torch.arange(1, g - case["empty"] + 1, device="cuda", dtype=torch.float32).reciprocal()
    order = torch.randperm(g - case["empty"], generator=gen, device="cuda")
    group_of = torch.multinomial(weight, nodes, replacement=True, generator=gen)
    group_of = order[group_of].to(torch.int32)
    group_of[torch.rand(nodes, generator=gen, device="cuda") < case["left_out"]] = -1
    return group_of, torch.randperm(nodes, generator=gen, device="cuda")[:n].to(torch.int32)


def prepare(case, seed):
    gen = _generator(seed)
    dtype = TYPES[case["dtype"]]
    if case["kind"] == "orthogonal":
        shape = (case["batch"], case["rows"], case["cols"])
        # a gradient: a few strong directions over a broad rest
        left = _normal(gen, shape[:2] + (4,), torch.float32)
        right = _normal(gen, (shape[0], 4, shape[2]), torch.float32, 0.5)
        update = (torch.randn(shape, generator=gen, device="cuda") + left @ right).mul_(1e-3).to(dtype)
        s = dict(case=case, dtype=dtype, update=update)
        if own:
            from paper_2112_08541_amd import binding as B
            s["plan"] = B.Orthogonalizer(*shape, dtype=dtype, steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
            s["out"] = torch.empty_like(update)
        return s
    s = _layer(case, gen)
    if case["kind"] == "grouped":
        s["group_of"], s["ids"] = _types(case, gen)
    if own:
        from paper_2112_08541_amd import binding as B
        n, k, m = case["rows"], case["in_dim"], case["out_dim"]
        groups = case.get("groups", 0)
        s["layer"] = B.Linear(n, k, m, dtype=dtype, activation=case["activation"], residual=case["residual"], num_groups=groups)
        s["sorted"] = B.RowGroups(n, groups) if groups else None
        s["y"] = torch.empty((n, m), dtype=dtype, device="cuda")
        if case["train"]:
            s["saved"] = torch.empty_like(s["y"]) if case["activation"] != "none" else None
            s["dx"] = torch.empty((n, k), dtype=dtype, device="cuda")
            s["dweight"] = torch.empty_like(s["weight"])
            s["dbias"] = torch.empty_like(s["bias"]) if case["bias"] else None
            s["dresidual"] = torch.empty_like(s["y"]) if case["residual"] == "before" else None
    return s


# ------------------------------------------------------------------ the framework's operators
def _run_own(s):
    case = s["case"]
    if case["kind"] == "orthogonal":
        s["plan"].run(s["update"], s["out"])
        return s["out"]
    out, groups = {}, s["sorted"]
    if groups is not None:
        groups.build(s["group_of"], ids=s["ids"])
        out.update(rows=groups.rows, offsets=groups.offsets)
    s["layer"].forward(s["x"], s["weight"], s["y"], bias=s["bias"], residual=s["residual"], saved=s.get("saved"), groups=groups)
    out["y"] = s["y"]
    if case["train"]:
        s["layer"].backward(s["dy"], s["x"], s["weight"], saved=s["saved"], dx=s["dx"], dweight=s["dweight"],
                            dbias=s["dbias"], dresidual=s["dresidual"], groups=groups)
        out.update(dx=s["dx"], dweight=s["dweight"])
        if case["bias"]:
            out["dbias"] = s["dbias"]
        if case["residual"] == "before":
            out["dresidual"] = s["dresidual"]
    return out


# ------------------------------------------------------------------ plain forms
def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(name, z, dy):
    if name == "relu":
        return torch.where(z > 0, dy, 0)
    if name == "gelu":
        return dy * (0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    if name == "silu":
        p = torch.sigmoid(z)
        return dy * (p * (1 + z * (1 - p)))
    return dy


def _orthogonal(update, steps):
    a, b, c = COEFFICIENTS
    x = update.float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    x = x.mT.contiguous() if tall else x
    for _ in range(steps):
        p = x @ x.mT.contiguous()
        x = a * x + (b * p + c * (p @ p)) @ x
    return (x.mT if tall else x).to(update.dtype).contiguous()


def _run_plain(s):
    case, dtype = s["case"], s["dtype"]
    if case["kind"] == "orthogonal":
        return _orthogonal(s["update"], case["steps"])
    out = {}
    grouped = case["kind"] == "grouped"
    x, w = s["x"].float(), s["weight"].float()
    if grouped:
        g = case["groups"]
        t = s["group_of"][s["ids"].long()]
        t = torch.where((t >= 0) & (t < g), t, g)                  # rows without a type come last
        rows = torch.argsort(t, stable=True)
        offsets = torch.zeros(g + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = torch.cumsum(torch.bincount(t, minlength=g + 1)[:g], 0)
        out.update(rows=rows.to(torch.int32), offsets=offsets)
        ends = offsets.tolist()
        sizes = [j - i for i, j in zip(ends, ends[1:])]
        typed = rows[: ends[-1]]
        parts = x[typed].split(sizes)
        z = torch.zeros((case["rows"], case["out_dim"]), device="cuda")
        z[typed] = torch.cat([p @ wg.t() for p, wg in zip(parts, w)])
        if case["bias"]:
            z[typed] += s["bias"].float()[t[typed].long()]
    else:
        z = x @ w.t()
        if case["bias"]:
            z += s["bias"].float()
    if case["residual"] == "before":
        z += s["residual"].float()
    y = _act(case["activation"], z)
    if case["residual"] == "after":
        y = y + s["residual"].float()
    out["y"] = y.to(dtype)
    if not case["train"]:
        return out
    dz = _act_grad(case["activation"], z, s["dy"].float())
    if grouped:
        up = dz[typed].split(sizes)
        dx = torch.zeros((case["rows"], case["in_dim"]), device="cuda")
        dx[typed] = torch.cat([d @ wg for d, wg in zip(up, w)])
        dw = torch.stack([d.t() @ p for d, p in zip(up, parts)])
        db = torch.stack([d.sum(0) for d in up]) if case["bias"] else None
    else:
        dx, dw = dz @ w, dz.t() @ x
        db = dz.sum(0) if case["bias"] else None
    out.update(dx=dx.to(dtype), dweight=dw.to(dtype))
    if case["bias"]:
        out["dbias"] = db.to(dtype)
    if case["residual"] == "before":
        out["dresidual"] = dz.to(dtype)
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    es = TYPES[case["dtype"]].itemsize
    if case["kind"] == "orthogonal":
        # each input once, each output once; two of a step's three products are symmetric: half of each is enough
        m, n = sorted((case["rows"], case["cols"]))
        return {"bytes": 2 * es * case["batch"] * m * n,
                "flops": case["steps"] * case["batch"] * (m * m * n + m * m * m + 2 * m * m * n)}
    n, k, m = case["rows"], case["in_dim"], case["out_dim"]
    g = case.get("groups", 1)
    weights = g * m * k + (g * m if case["bias"] else 0)
    values = n * k + n * m + weights + (n * m if case["residual"] != "none" else 0)
    if case["train"]:
        values += n * m + n * k + weights + (n * m if case["residual"] == "before" else 0)
    extra = 4 * (3 * n + g + 1) if case["kind"] == "grouped" else 0        # ids, their types, the sorted rows
    return {"bytes": es * values + extra, "flops": (6 if case["train"] else 2) * n * k * m}


# ------------------------------------------------------------------ the definition in 64 bits
def _phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "orthogonal":
        # The steps act on the singular values alone: X -> X q(X'X) with q(t) = a + b t + c t^2, t a squared singular value.
        a, b, c = COEFFICIENTS
        u = s["update"].double().cpu().numpy()
        outs = []
        for one in u:
            one = one / (np.sqrt((one * one).sum()) + EPS)
            left = one.shape[0] <= one.shape[1]
            t, v = np.linalg.eigh(one @ one.T if left else one.T @ one)
            factor = np.ones_like(t)
            for _ in range(case["steps"]):
                q = a + b * t + c * t * t
                factor, t = factor * q, t * q * q
            poly = (v * factor) @ v.T
            outs.append(poly @ one if left else one @ poly)
        return torch.from_numpy(np.stack(outs))
    n, m, k = case["rows"], case["out_dim"], case["in_dim"]
    x, w = s["x"].double(), s["weight"].double()
    b = s["bias"].double() if case["bias"] else None
    res = s["residual"].double() if case["residual"] != "none" else None
    grouped = case["kind"] == "grouped"
    if grouped:
        t = s["group_of"][s["ids"].long()]
        members = [torch.nonzero(t == i).squeeze(1) for i in range(case["groups"])]
    else:
        w, b = w[None], None if b is None else b[None]
        members = [torch.arange(n, device="cuda")]
    z = torch.zeros((n, m), dtype=torch.float64, device="cuda") if res is None or case["residual"] == "after" else res.clone()
    for i, at in enumerate(members):
        z[at] += torch.mm(x[at], w[i].t().contiguous()) + (0 if b is None else b[i])
    name = case["activation"]
    if name == "relu":
        y, slope = z * (z > 0), (z > 0).double()
    elif name == "gelu":
        y, slope = z * _phi(z), _phi(z) + z * torch.exp(-z * z / 2) * (2 * math.pi) ** -0.5
    elif name == "silu":
        e = torch.exp(-z)
        y, slope = z / (1 + e), (1 + e + z * e) / (1 + e) ** 2
    else:
        y, slope = z, torch.ones_like(z)
    out = {"y": y + res if case["residual"] == "after" else y}
    if grouped:
        out.update(rows=None, offsets=None)
    if case["train"]:
        dz = s["dy"].double() * slope
        dx = torch.zeros((n, k), dtype=torch.float64, device="cuda")
        dw, db = torch.zeros_like(w), torch.zeros((len(members), m), dtype=torch.float64, device="cuda")
        for i, at in enumerate(members):
            dx[at] = torch.mm(dz[at], w[i])
            dw[i] = torch.mm(dz[at].t().contiguous(), x[at])
            db[i] = dz[at].sum(0)
        out.update(dx=dx, dweight=dw if grouped else dw[0])
        if case["bias"]:
            out["dbias"] = db if grouped else db[0]
        if case["residual"] == "before":
            out["dresidual"] = dz
    return out
