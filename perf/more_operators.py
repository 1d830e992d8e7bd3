"""The operators between a model's last hidden rows and its update: what is measured of them.

The rows are those of a batch's nodes (any hop's for the norm, the seeds' for the losses), fp32 or bf16.
  norm      layer norm over each row, and with `train` its gradients, those of weight and bias summed over all rows
  labels    softmax cross entropy of class scores x W' + b that are not kept, and with `train` its gradients
  distill   the same scores against a teacher's top classes at a temperature, alone or beside the labels, with gradients

The plain forms below are elementary torch operations in 32 bits; `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # One node's prediction: a single row, where the call itself is the cost.
        dict(name="norm one row", kind="norm", dtype="bf16", rows=1, width=512, affine=True, train=False),
        # A training step of the norm over a small batch's nodes.
        dict(name="norm small train", kind="norm", dtype="f32", rows=5_485, width=100, affine=True, train=True),
        # A training step of the norm behind the input layer of an ordinary batch, fp32.
        dict(name="norm train f32", kind="norm", dtype="f32", rows=428_377, width=256, affine=True, train=True),
        # The same over the wide bf16 rows.
        dict(name="norm train bf16", kind="norm", dtype="bf16", rows=302_709, width=512, affine=True, train=True),
        # One node's loss over very many classes: the weight is what has to be read.
        dict(name="labels one row", kind="labels", dtype="bf16", rows=1, in_dim=512, classes=65_536, train=False),
        # A training step over a batch's seeds and a few dozen classes, fp32.
        dict(name="labels few classes train", kind="labels", dtype="f32", rows=1_024, in_dim=128, classes=50, train=True),
        # The loss of all training nodes at the end of an epoch, forward only.
        dict(name="labels evaluation", kind="labels", dtype="bf16", rows=204_800, in_dim=256, classes=150, train=False),
        # A training step with a class for every item of a catalogue, fp32, an odd number of them.
        dict(name="labels train f32", kind="labels", dtype="f32", rows=1_024, in_dim=256, classes=50_001, train=True),
        # The same for a wide batch's seeds in bf16.
        dict(name="labels train bf16", kind="labels", dtype="bf16", rows=4_096, in_dim=512, classes=65_536, train=True),
        # A small student beside its labels, a teacher's eight best classes of each seed.
        dict(name="distill small train", kind="distill", dtype="f32", rows=512, in_dim=100, classes=150, top=8,
             temperature=2.0, labels=True, train=True),
        # The teacher's loss alone of a large set of nodes, forward only.
        dict(name="distill evaluation", kind="distill", dtype="bf16", rows=50_000, in_dim=256, classes=1_001, top=16,
             temperature=3.0, labels=False, train=False),
        # A training step on a teacher's many best classes and the labels, a class for every item.
        dict(name="distill train bf16", kind="distill", dtype="bf16", rows=4_096, in_dim=512, classes=40_003, top=32,
             temperature=1.5, labels=True, train=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "labels", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    train = rng.random() < 0.6
    if kind == "norm":
        width = _log_int(rng, 8, 8192)
        most = min(428_377, (110_000_000 if dtype == "f32" else 154_000_000) // width)
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, most), width=width, affine=rng.random() < 0.75, train=train)
    in_dim, classes = _log_int(rng, 8, 640), _log_int(rng, 2, 65_536)
    # no more products, and no more scores in the plain form, than the largest listed case of the type
    most = (13_000_000_000 if dtype == "f32" else 137_000_000_000) // (in_dim * classes)
    most = max(1, min(most, (51_000_000 if dtype == "f32" else 160_000_000) // classes, 50_000_000 // in_dim, 204_800))
    case = dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, most), in_dim=in_dim, classes=classes, train=train)
    if kind == "distill":
        case.update(top=_log_int(rng, 1, min(64, classes)), temperature=rng.choice([1.0, 1.5, 2.0, 4.0]), labels=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 1)
    return g


def _normal(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale)


def _rows_to_normalise(case, gen, dtype):
    """Rows whose means and spreads differ, some columns larger than others."""
    n, w = case["rows"], case["width"]
    spread = torch.exp(_normal(gen, (n, 1), 0.5))
    columns = torch.exp(_normal(gen, (1, w), 0.5))
    return (_normal(gen, (n, w)) * columns + _normal(gen, (n, 1))).mul_(spread).to(dtype)


def _labelled_rows(case, gen, dtype):
    """Hidden rows, the head, and labels that a half-trained head gives some of its belief to; one row in twenty has none."""
    n, d, v = case["rows"], case["in_dim"], case["classes"]
    weight = _normal(gen, (v, d), 1.5 / math.sqrt(d))
    bias = _normal(gen, (v,), 0.5)
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    x = _normal(gen, (n, d)) + 2.0 * weight[labels.long()]
    labels[torch.rand(n, generator=gen, device="cuda") < 0.05] = -1
    return x.to(dtype), weight.to(dtype), bias.to(dtype), labels


def _teacher(case, gen, labels):
    """A row's `top` classes, best first, all different, and their scores; some rows have fewer (the rest -1), a few none."""
    n, v, k = case["rows"], case["classes"], case["top"]
    first = torch.where(labels >= 0, labels, 0).long()[:, None]
    # classes a random step apart from each other, round the classes from the label on
    step = v // k
    jump = torch.randint(0, max(step, 1), (n, k), generator=gen, device="cuda")
    jump[:, 0] = 0
    classes = (first + torch.arange(k, device="cuda") * step + jump) % v
    scores = _normal(gen, (n, k), 2.0).sort(dim=1, descending=True).values + 3.0
    have = torch.randint(1, k + 1, (n, 1), generator=gen, device="cuda")
    have = torch.where(torch.rand((n, 1), generator=gen, device="cuda") < 0.9, k, have)
    have = torch.where(torch.rand((n, 1), generator=gen, device="cuda") < 0.03, 0, have)
    classes = torch.where(torch.arange(k, device="cuda") < have, classes, -1)
    return classes.to(torch.int32), scores


def prepare(case, seed):
    gen = _generator(seed)
    dtype = TYPES[case["dtype"]]
    n = case["rows"]
    s = dict(case=case, dtype=dtype)
    if case["kind"] == "norm":
        w = case["width"]
        s["x"] = _rows_to_normalise(case, gen, dtype)
        s["weight"] = (1.0 + _normal(gen, (w,), 0.2)).to(dtype) if case["affine"] else None
        s["bias"] = _normal(gen, (w,), 0.2).to(dtype) if case["affine"] else None
        s["dy"] = _normal(gen, (n, w)).to(dtype) if case["train"] else None
        if own:
            from paper_2112_08541_amd import binding as B
            s["norm"] = B.LayerNorm(n, w, dtype=dtype, eps=EPS)
            s["y"] = torch.empty_like(s["x"])
            if case["train"]:
                s["saved"] = torch.empty((n, 2), dtype=torch.float32, device="cuda")
                s["dx"] = torch.empty_like(s["x"])
                s["dweight"] = torch.empty_like(s["weight"]) if case["affine"] else None
                s["dbias"] = torch.empty_like(s["bias"]) if case["affine"] else None
        return s
    s["x"], s["weight"], s["bias"], s["labels"] = _labelled_rows(case, gen, dtype)
    distill = case["kind"] == "distill"
    s["teacher"] = _teacher(case, gen, s["labels"]) if distill else None
    if distill and not case["labels"]:
        s["labels"] = None
    if own:
        from paper_2112_08541_amd import binding as B
        s["head"] = B.ClassLoss(n, case["in_dim"], case["classes"], dtype=dtype, top=case.get("top", 0),
                                temperature=case.get("temperature", 1.0))
        s["loss"] = torch.empty(n, dtype=torch.float32, device="cuda") if s["labels"] is not None else None
        s["teacher_loss"] = torch.empty(n, dtype=torch.float32, device="cuda") if distill else None
        if case["train"]:
            s["saved"] = torch.empty((n, s["head"].saved_width), dtype=torch.float32, device="cuda")
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"] = torch.empty_like(s["weight"])
            s["dbias"] = torch.empty_like(s["bias"])
    return s


def _shares(case):
    """What a row's two losses count in the mean that is differentiated."""
    if case["kind"] == "labels":
        return 1.0 / case["rows"], 0.0
    return (0.4 / case["rows"], 0.6 / case["rows"]) if case["labels"] else (0.0, 1.0 / case["rows"])


# ------------------------------------------------------------------ the framework's operators
def _run_own(s):
    case = s["case"]
    if case["kind"] == "norm":
        s["norm"].forward(s["x"], s["y"], weight=s["weight"], bias=s["bias"], saved=s.get("saved"))
        out = {"y": s["y"]}
        if case["train"]:
            s["norm"].backward(s["dy"], s["x"], s["saved"], weight=s["weight"], dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"])
            out["dx"] = s["dx"]
            if case["affine"]:
                out.update(dweight=s["dweight"], dbias=s["dbias"])
        return out
    s["head"].forward(s["x"], s["weight"], bias=s["bias"], labels=s["labels"], teacher=s["teacher"], loss=s["loss"],
                      teacher_loss=s["teacher_loss"], saved=s.get("saved"))
    out = {}
    if s["loss"] is not None:
        out["loss"] = s["loss"]
    if s["teacher_loss"] is not None:
        out["teacher_loss"] = s["teacher_loss"]
    if case["train"]:
        share, teacher_share = _shares(case)
        s["head"].backward(s["x"], s["weight"], s["saved"], bias=s["bias"], labels=s["labels"], teacher=s["teacher"], scale=share,
                           teacher_scale=teacher_share, dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"])
        out.update(dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"])
    return out


# ------------------------------------------------------------------ plain forms
def _plain_norm(s):
    case, dtype = s["case"], s["dtype"]
    x = s["x"].float()
    weight = s["weight"].float() if case["affine"] else None
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    scale = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
    hat = centred * scale
    y = hat * weight + s["bias"].float() if case["affine"] else hat
    out = {"y": y.to(dtype)}
    if case["train"]:
        dy = s["dy"].float()
        g = dy * weight if case["affine"] else dy
        dx = scale * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
        out["dx"] = dx.to(dtype)
        if case["affine"]:
            out.update(dweight=(dy * hat).sum(0).to(dtype), dbias=dy.sum(0).to(dtype))
    return out


def _softmax_parts(z):
    """exp(z) over its row's sum, and the logarithm of that sum."""
    most = z.max(1, keepdim=True).values
    e = (z - most).exp()
    total = e.sum(1, keepdim=True)
    return e.div_(total), most + total.log()


def _run_plain(s):
    case, dtype = s["case"], s["dtype"]
    if case["kind"] == "norm":
        return _plain_norm(s)
    x, w = s["x"].float(), s["weight"].float()
    z = x @ w.t()
    z += s["bias"].float()
    at = torch.arange(case["rows"], device="cuda")
    share, teacher_share = _shares(case)
    out, dz = {}, None
    if s["labels"] is not None:
        have = s["labels"] >= 0
        label = torch.where(have, s["labels"], 0).long()
        q, lse = _softmax_parts(z)
        out["loss"] = torch.where(have, lse[:, 0] - z[at, label], 0.0)
        if case["train"]:
            q[at, label] -= 1.0
            dz = torch.where(have[:, None], q * share, 0.0)
        del q
    if case["kind"] == "distill":
        t = case["temperature"]
        classes, scores = s["teacher"]
        have = classes >= 0
        some = have.any(1)
        place = torch.where(have, classes, 0).long()
        top = torch.where(have, scores / t, -math.inf)
        best = torch.where(some, top.max(1).values, 0.0)[:, None]
        p = (top - best).exp()
        total = torch.where(some, p.sum(1), 1.0)[:, None]
        p = p / total
        logp = torch.where(have, top - best - total.log(), 0.0)
        q, lse = _softmax_parts(z / t)
        out["teacher_loss"] = torch.where(some, t * t * (p * (logp - z.gather(1, place) / t + lse)).sum(1), 0.0)
        if case["train"]:
            d = q.scatter_add_(1, place, -p)
            d = torch.where(some[:, None], d * (t * teacher_share), 0.0)
            dz = d if dz is None else dz + d
    if case["train"]:
        out.update(dx=(dz @ w).to(dtype), dweight=(dz.t() @ x).to(dtype), dbias=dz.sum(0).to(dtype))
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    es = TYPES[case["dtype"]].itemsize
    n, train = case["rows"], case["train"]
    if case["kind"] == "norm":
        w = case["width"]
        values = (4 if train else 2) * n * w + ((4 if train else 2) * w if case["affine"] else 0)
        return {"bytes": es * values, "flops": (18 if train else 7) * n * w}
    d, v = case["in_dim"], case["classes"]
    values = n * d + v * d + v
    outputs = n * d + v * d + v if train else 0
    with_labels = case["kind"] == "labels" or case["labels"]
    extra = (8 * n if with_labels else 0) + (n * (8 * case["top"] + 4) if case["kind"] == "distill" else 0)
    return {"bytes": es * (values + outputs) + extra, "flops": (6 if train else 2) * n * d * v}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_norm(s):
    case = s["case"]
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    deviation = torch.sqrt(var + EPS)
    hat = (x - mean) / deviation
    gamma = s["weight"].double() if case["affine"] else torch.ones(case["width"], dtype=torch.float64, device="cuda")
    beta = s["bias"].double() if case["affine"] else torch.zeros_like(gamma)
    out = {"y": torch.addcmul(beta, hat, gamma)}
    if case["train"]:
        dy = s["dy"].double()
        # the gradient is g without its parts along the row of ones and along hat
        g = dy * gamma
        g = g - g.sum(1, keepdim=True) / case["width"]
        along = torch.mul(g, hat).sum(1, keepdim=True) / case["width"]
        out["dx"] = torch.addcmul(g, along, hat, value=-1.0) / deviation
        if case["affine"]:
            out["dweight"] = torch.mul(dy, hat).sum(0)
            out["dbias"] = dy.sum(0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    n, v = case["rows"], case["classes"]
    weight, bias = s["weight"].double(), s["bias"].double()
    share, teacher_share = _shares(case)
    distill = case["kind"] == "distill"
    parts = {"loss": [], "teacher_loss": [], "dx": []}
    dweight = torch.zeros_like(weight)
    dbias = torch.zeros_like(bias)
    step = max(1, 60_000_000 // v)
    for first in range(0, n, step):
        rows = slice(first, min(n, first + step))
        x = s["x"][rows].double()
        z = torch.addmm(bias, x, weight.t().contiguous())
        dz = torch.zeros_like(z) if case["train"] else None
        if s["labels"] is not None:
            labels = s["labels"][rows]
            named = torch.nonzero(labels >= 0).squeeze(1)
            logq = torch.log_softmax(z[named], 1)
            label = labels[named].long()[:, None]
            loss = torch.zeros(len(labels), dtype=torch.float64, device="cuda")
            loss[named] = -logq.gather(1, label)[:, 0]
            parts["loss"].append(loss)
            if case["train"]:
                one = torch.zeros_like(logq).scatter_(1, label, 1.0)
                dz[named] += share * (logq.exp() - one)
        if distill:
            t = case["temperature"]
            classes, scores = s["teacher"][0][rows], s["teacher"][1][rows].double()
            taught = torch.nonzero((classes >= 0).any(1)).squeeze(1)
            chosen = classes[taught]
            belief = torch.softmax(scores[taught].masked_fill(chosen < 0, -math.inf) / t, 1)
            target = torch.zeros((len(taught), v), dtype=torch.float64, device="cuda")
            target.scatter_add_(1, chosen.clamp(min=0).long(), belief)
            logq = torch.log_softmax(z[taught] / t, 1)
            loss = torch.zeros(len(classes), dtype=torch.float64, device="cuda")
            loss[taught] = t * t * (torch.special.xlogy(belief, belief).sum(1) - (target * logq).sum(1))
            parts["teacher_loss"].append(loss)
            if case["train"]:
                dz[taught] += t * teacher_share * (logq.exp() - target)
        if case["train"]:
            parts["dx"].append(torch.mm(dz, weight))
            dweight += torch.mm(dz.t().contiguous(), x)
            dbias += dz.sum(0)
    out = {k: torch.cat(p) for k, p in parts.items() if p}
    if case["train"]:
        out.update(dweight=dweight, dbias=dbias)
    return out
