"""Losses over class scores and their gradients against the definition in 64 bits.

u = 2^-24 is the unit roundoff of sums, v that of the type (2^-24 or 2^-8).  A score is a sum of D products of exact factors and the bias: off by Z = (D + 4) u
(sum|x||w| + |b|).  exp is right to 4 u and what its argument is off by: u (1 + 2 |argument|), which e^-a a <= 0.4 keeps below 1 u in a sum.  A sum of exp has at most 16 + 2 +
2 + classes / 8192 + 1 + 6 steps, each rescaling a partial sum by another exp (8 u): together less than S = (120 + classes / 1000) u of itself, and the logarithm adds 4 u of its value.
So the logarithm of the sum is off by max Z + S + 4 u |log sum| + 2 u max|z|, and each loss by that, Z of its own score and its own roundings.
dz = s (q - onehot) + t s' (q_t - p): each q off by q (Z + that + 8 u (1 + |argument|)), p by p (12 u + 2 u |argument|) and the sum's; dz is rounded to the type.  The
products add (terms + 8) u of the absolute products, and the result is rounded."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
V = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


@pytest.fixture(scope="module")
def B(torch):
    from paper_2112_08541_amd import binding
    binding.lib()
    return binding


def dtype_of(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


class Reference:
    """In 64 bits on the GPU, every value with its bound."""

    def __init__(self, torch, x, w, b, labels, teacher, t, v):
        self.torch, self.v, self.t = torch, v, t
        self.x, self.w = x.double(), w.double()
        n, D = x.shape
        self.C = C = w.shape[0]
        bias = torch.zeros(C, dtype=torch.float64, device="cuda") if b is None else b.double()
        self.z = self.x @ self.w.t().contiguous() + bias
        size = self.x.abs() @ self.w.abs().t().contiguous() + torch.nan_to_num(bias.abs(), posinf=0.0)
        self.Z = (D + 4) * U * size
        self.big = torch.where(self.z.isinf(), 0.0, self.z.abs()).max(1, keepdim=True).values
        self.worst = self.Z.max(1, keepdim=True).values
        self.sum = (120 + C / 1000) * U
        at = torch.arange(n, device="cuda")
        if labels is not None:
            self.have = (labels >= 0) & (labels < C)
            self.label = torch.where(self.have, labels, 0).long()
            lse = torch.logsumexp(self.z, 1, keepdim=True)
            self.q, self.lse_off = (self.z - lse).exp(), self.worst + self.sum + 4 * U * lse.abs() + 2 * U * self.big
            self.arg = self.z - lse
            own = self.z[at, self.label]
            self.loss = torch.where(self.have, lse[:, 0] - own, 0.0)
            self.loss_bound = self.lse_off[:, 0] + self.Z[at, self.label] + 4 * U * (self.loss.abs() + self.big[:, 0])
        if teacher is not None:
            classes, scores = teacher[0].long(), teacher[1].double() / t
            have = (classes >= 0) & (classes < C)
            self.place = torch.where(have, classes, 0)
            top = torch.where(have, scores, -np.inf)
            self.some = (top > -np.inf).any(1)
            best = torch.where(self.some, top.max(1).values, 0.0)[:, None]
            e = (top - best).exp()
            total = torch.where(self.some, e.sum(1), 1.0)[:, None]
            self.p = e / total
            far = torch.nan_to_num((top - best).abs(), posinf=0.0)
            self.p_off = self.p * (40 + scores.shape[1]) * U + self.p * U * (4 * far + 3 * torch.nan_to_num(scores.abs(), posinf=0.0))
            lse = torch.logsumexp(self.z / t, 1, keepdim=True)
            self.qt, self.arg_t = (self.z / t - lse).exp(), self.z / t - lse
            self.lse_t_off = self.worst / t + self.sum + 4 * U * lse.abs() + 3 * U * self.big / t
            logp = torch.where(self.p > 0, top - best - total.log(), 0.0)
            logq = torch.where(self.p > 0, self.arg_t.gather(1, self.place), 0.0)
            self.teacher_loss = torch.where(self.some, t * t * (self.p * (logp - logq)).sum(1), 0.0)
            each = self.Z.gather(1, self.place) / t + self.lse_t_off + 8 * U * (logp.abs() + logq.abs() + 3 * torch.nan_to_num(scores.abs(), posinf=0.0) + self.big / t) + 50 * U
            self.teacher_bound = t * t * (self.p * each + (self.p_off + scores.shape[1] * U * self.p) * (logp - logq).abs()).sum(1) + 2 * U * self.teacher_loss.abs()

    def gradients(self, s, st):
        torch, v = self.torch, self.v
        dz, off = torch.zeros_like(self.z), torch.zeros_like(self.z)
        if hasattr(self, "q") and s:
            d = self.q.clone()
            d[torch.arange(len(d), device="cuda"), self.label] -= 1.0
            e = self.q * (self.Z + self.lse_off + 8 * U * (1 + torch.nan_to_num(self.arg.abs(), posinf=0.0))) + 2 * U * d.abs()
            dz += torch.where(self.have[:, None], s * d, 0.0)
            off += torch.where(self.have[:, None], abs(s) * e, 0.0)
        if hasattr(self, "qt") and st:
            d = self.qt.clone().scatter_add_(1, self.place, -self.p)
            e = self.qt * (self.Z / self.t + self.lse_t_off + 8 * U * (1 + torch.nan_to_num(self.arg_t.abs(), posinf=0.0)))
            e = e.scatter_add_(1, self.place, self.p_off + 4 * U * self.p) + 4 * U * d.abs()
            dz += torch.where(self.some[:, None], self.t * st * d, 0.0)
            off += torch.where(self.some[:, None], self.t * abs(st) * e, 0.0)
        off += 1.01 * v * dz.abs() + 1e-40
        off += off * v
        out = []
        for value, size, spread, terms in ((dz @ self.w, dz.abs() @ self.w.abs(), off @ self.w.abs(), self.C), (dz.t().contiguous() @ self.x, dz.abs().t().contiguous() @ self.x.abs(), off.t().contiguous() @ self.x.abs(), len(dz)),
                                           (dz.sum(0), dz.abs().sum(0), off.sum(0), len(dz))):
            out.append((value, (terms + 8) * U * (size + spread) + spread + 1.01 * v * (value.abs() + spread) + 1e-37))
        return out


def check(name, got, want, bound):
    over = (got.double() - want).abs() - bound
    assert got.isfinite().all(), name
    assert (over <= 0).all(), f"{name}: {float((got.double() - want).abs().max())} off, worst {float(over.max())} beyond its bound at {int(over.argmax())} of {tuple(got.shape)}"


def inputs(torch, kind, n, D, C, k, seed, pad=0, bias=True, scale=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = dtype_of(torch, kind)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    x = torch.cat([rnd(n, D), torch.full((n, pad), float("nan"), device="cuda")], 1).to(t)[:, :D]
    w, b = (rnd(C, D) * scale / D ** 0.5).to(t), (rnd(C) * 0.5).to(t) if bias else None
    labels = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
    teacher = None
    if k:
        classes = torch.randint(0, C, (n, k), generator=g, device="cuda", dtype=torch.int32)      # (the same class now and then)
        classes[torch.rand((n, k), generator=g, device="cuda") < 0.1] = -1
        classes[torch.rand(n, generator=g, device="cuda") < 0.1] = C + 3
        teacher = (classes, rnd(n, k) * 2)
        if n > 2:
            teacher[0][n // 2, 0] = labels[n // 2]
    return x, w, b, labels, teacher


def run(torch, B, kind, x, w, b, labels, teacher, t=1.0, s=0.0, st=0.0, want=("dx", "dweight", "dbias"), head=None, stream=None):
    n, D = x.shape
    C, ty = w.shape[0], dtype_of(torch, kind)
    head = head or B.ClassLoss(n, D, C, ty, top=0 if teacher is None else teacher[0].shape[1], temperature=t)
    new = lambda *shape, ty=torch.float32: torch.full(shape, 7.0, dtype=ty, device="cuda")      # noqa: E731
    out = dict(saved=new(n, head.saved_width), dx=new(n, D, ty=ty), dweight=new(C, D, ty=ty), dbias=new(C, ty=ty))
    out["loss"] = None if labels is None else new(n)
    out["teacher_loss"] = None if teacher is None else new(n)
    head.forward(x, w, bias=b, labels=labels, teacher=teacher, loss=out["loss"], teacher_loss=out["teacher_loss"], saved=out["saved"], stream=stream)
    head.backward(x, w, out["saved"], bias=b, labels=labels, teacher=teacher, scale=s, teacher_scale=st, stream=stream, **{k: out[k] for k in want})
    return out


def check_all(torch, B, kind, data, t=1.0, s=0.3, st=0.7):
    x, w, b, labels, teacher = data
    ref = Reference(torch, x, w, b, labels, teacher, t, V[kind])
    got = run(torch, B, kind, x, w, b, labels, teacher, t, s, st)
    if labels is not None:
        check("loss", got["loss"], ref.loss, ref.loss_bound)
    if teacher is not None:
        check("teacher_loss", got["teacher_loss"], ref.teacher_loss, ref.teacher_bound)
    for name, (value, bound) in zip(("dx", "dweight", "dbias"), ref.gradients(s, st)):
        check(name, got[name], value, bound)
    return got


SHAPES = [(1, 1, 1), (1, 5, 2), (3, 7, 3), (2, 8, 17), (15, 16, 16), (16, 33, 50), (17, 100, 127), (63, 64, 128), (64, 9, 129), (65, 31, 130), (100, 128, 255), (129, 130, 257), (37, 257, 511), (40, 500, 1_030),
          (130, 64, 150), (300, 100, 50), (7, 640, 2_000), (600, 72, 384), (33, 512, 3_001)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C", SHAPES)
def test_labels(torch, B, kind, n, D, C):
    x, w, b, labels, _ = inputs(torch, kind, n, D, C, 0, seed=n + C, pad=3 if n % 2 else 0, bias=C % 3 > 0)
    check_all(torch, B, kind, (x, w, b, labels, None), s=1.0 / n, st=0.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C", SHAPES)
def test_a_teacher_alone_and_beside_labels(torch, B, kind, n, D, C):
    k = min(C, 1 + (n * 7 + C) % 9)
    data = inputs(torch, kind, n, D, C, k, seed=n + C + 1)
    check_all(torch, B, kind, data, t=2.0, s=0.4 / n, st=0.6 / n)
    check_all(torch, B, kind, (*data[:3], None, data[4]), t=1.0, s=0.0, st=1.0 / n)


@pytest.mark.parametrize("k,t", [(1, 4.0), (64, 0.5), (65, 3.0), (200, 1.5), (1024, 8.0)])
def test_many_classes_of_the_teacher(torch, B, k, t):
    check_all(torch, B, "f32", inputs(torch, "f32", 21, 40, 1_500, k, seed=k), t=t)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [(1_500, 100, 10, 0), (3_000, 24, 700, 4), (40_000, 8, 3, 2), (1_100, 128, 4_000, 8), (2_100, 16, 16_390, 3), (20_000, 8, 1_700, 0), (17_000, 8, 16_400, 2), (5_000, 136, 7_000, 0)])
def test_pieces_and_shares(torch, B, kind, n, D, C, k):
    """Sizes at which dz is made in several pieces of rows, of classes or of both, and products share the summed index."""
    data = inputs(torch, kind, n, D, C, k, seed=n)
    got = check_all(torch, B, kind, data, t=2.0, s=1.0 / n, st=1.0 / n if k else 0.0)
    again = run(torch, B, kind, *data, 2.0, 1.0 / n, 1.0 / n if k else 0.0)
    assert all(torch.equal(got[i], again[i]) for i in got if got[i] is not None)
    half = run(torch, B, kind, *data, 2.0, 1.0 / n, 1.0 / n if k else 0.0, want=("dx",))
    assert torch.equal(half["dx"], got["dx"]) and (half["dweight"] == 7).all() and (half["dbias"] == 7).all()
    half = run(torch, B, kind, *data, 2.0, 1.0 / n, 1.0 / n if k else 0.0, want=("dweight",))
    assert torch.equal(half["dweight"], got["dweight"]) and (half["dx"] == 7).all() and (half["dbias"] == 7).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scores_that_differ_much(torch, B, kind):
    """Classes with a probability of 1e-12 and less: their gradients are right relative to themselves, and losses near 0 and near 100 are."""
    x, w, b, labels, teacher = inputs(torch, kind, 90, 60, 300, 5, seed=77, scale=12.0)
    b[100:200] -= 30
    check_all(torch, B, kind, (x, w, b, labels, teacher), t=1.5)


def test_classes_taken_out_and_rows_that_are_not_finite(torch, B):
    x, w, b, labels, teacher = inputs(torch, "f32", 50, 20, 300, 3, seed=5)
    out = torch.zeros(300, dtype=torch.bool, device="cuda")
    out[:130], out[200:] = True, True
    b[out] = -float("inf")
    labels[:] = torch.randint(130, 200, (50,), device="cuda", dtype=torch.int32)
    labels[4] = -1
    teacher[0][:] = torch.randint(130, 200, (50, 3), device="cuda", dtype=torch.int32)
    teacher[1][7] = -float("inf")          # nothing to learn from
    teacher[1][8, 0] = -float("inf")       # one class less
    got = check_all(torch, B, "f32", (x, w, b, labels, teacher), t=2.0)
    assert (got["dweight"][out] == 0).all() and (got["dbias"][out] == 0).all() and got["teacher_loss"][7] == 0 and got["loss"][4] == 0
    labels[3] = 0                          # a class that was taken out
    assert run(torch, B, "f32", x, w, b, labels, None, s=1.0)["loss"][3] == float("inf")
    # rows without a label may hold anything
    labels[3] = 150
    clean = run(torch, B, "f32", x, w, b, labels, None, s=1.0)
    x2 = x.clone()
    x2[4] = float("nan")
    got = run(torch, B, "f32", x2, w, b, labels, None, s=1.0)
    for k in ("loss", "dx", "dweight", "dbias"):
        assert torch.equal(got[k], clean[k]), k
    # one that has a label spoils itself, and no other row's loss and dx
    x2[5, 3] = float("inf")
    got = run(torch, B, "f32", x2, w, b, labels, None, s=1.0)
    keep = [i for i in range(50) if i != 5]
    assert got["loss"][5].isnan() and got["dx"][5].isnan().all()
    assert torch.equal(got["loss"][keep], clean["loss"][keep]) and torch.equal(got["dx"][keep], clean["dx"][keep])


def test_no_row_has_a_label(torch, B):
    x, w, b, labels, teacher = inputs(torch, "bf16", 70, 40, 90, 3, seed=6)
    labels.fill_(-1)
    teacher[0].fill_(90)
    x[:] = float("nan")
    got = run(torch, B, "bf16", x, w, b, labels, teacher, 2.0, 1.0, 1.0)
    assert all((got[k] == 0).all() for k in ("loss", "teacher_loss", "dx", "dweight", "dbias"))


def test_no_rows(torch, B):
    head = B.ClassLoss(10, 20, 30)
    e, s, w = torch.empty((0, 20), device="cuda"), torch.empty((0, 2), device="cuda"), torch.zeros((30, 20), device="cuda")
    labels = torch.empty(0, dtype=torch.int32, device="cuda")
    dw, db = torch.full((30, 20), 7.0, device="cuda"), torch.full((30,), 7.0, device="cuda")
    head.forward(e, w, labels=labels, saved=s)
    head.backward(e, w, s, labels=labels, dx=e, dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


def test_gradients_are_differences(torch, B):
    x, w, b, labels, teacher = inputs(torch, "f32", 5, 4, 7, 3, seed=4)
    got = run(torch, B, "f32", x, w, b, labels, teacher, 2.0, 0.3, 0.7)

    def total(x, w, b):
        r = Reference(torch, x, w, b, labels, teacher, 2.0, 0.0)
        return float((0.3 * r.loss).sum() + (0.7 * r.teacher_loss).sum())
    step = 1e-5
    for name, at in (("dx", 0), ("dweight", 1), ("dbias", 2)):
        args = [t.double() for t in (x, w, b)]
        grad = torch.zeros_like(args[at])
        for i in np.ndindex(*grad.shape):
            keep = float(args[at][i])
            args[at][i] = keep + step
            up = total(*args)
            args[at][i] = keep - step
            grad[i] = (up - total(*args)) / (2 * step)
            args[at][i] = keep
        # central differences: step^2 times third derivatives (below 1e2), rounding 1e-15 / 1e-5; the kernel: fp32 sums of some values below 10
        torch.testing.assert_close(got[name].double(), grad, atol=2e-5, rtol=2e-5)


def test_one_object_for_fewer_rows(torch, B):
    """A workspace made for many rows, calls of fewer, beside one made for them."""
    for kind, D, C in (("f32", 30, 1_100), ("bf16", 200, 17_000)):
        head = B.ClassLoss(3_000, D, C, dtype_of(torch, kind), top=2, temperature=2.0)
        for n in (3_000, 1, 40, 1_030, 0, 2_048):
            data = inputs(torch, kind, n, D, C, 2, seed=n)
            got, want = (run(torch, B, kind, *data, 2.0, 0.1, 0.1, head=h) for h in (head, None))
            assert all(torch.equal(got[i], want[i]) for i in got), n


def test_offsets_beyond_32_bits(torch, B):
    n, stride, D = 1_100, 1 << 21, 24
    x, w, b, labels, _ = inputs(torch, "bf16", n, D, 40, 0, seed=9)
    room = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    far = room.view(n, stride)[:, :D]
    far.copy_(x)
    want = run(torch, B, "bf16", x, w, b, labels, None, s=0.1)
    got = run(torch, B, "bf16", far, w, b, labels, None, s=0.1)
    assert all(torch.equal(got[k], want[k]) for k in ("loss", "dx", "dweight", "dbias"))
    head = B.ClassLoss(n, D, 40, torch.bfloat16)
    head.backward(x, w, want["saved"], bias=b, labels=labels, scale=0.1, dx=far)
    assert torch.equal(far, want["dx"])


def test_graph_and_other_stream(torch, B):
    make = lambda seed: inputs(torch, "bf16", 700, 96, 1_300, 4, seed=seed)      # noqa: E731
    x, w, b, labels, teacher = make(1)
    head = B.ClassLoss(700, 96, 1_300, torch.bfloat16, top=4, temperature=2.0)
    out = {}

    def both(stream=None):
        head.forward(x, w, bias=b, labels=labels, teacher=teacher, loss=out["loss"], teacher_loss=out["teacher_loss"], saved=out["saved"], stream=stream)
        head.backward(x, w, out["saved"], bias=b, labels=labels, teacher=teacher, scale=0.4, teacher_scale=0.6, dx=out["dx"], dweight=out["dweight"], dbias=out["dbias"], stream=stream)
    want = run(torch, B, "bf16", x, w, b, labels, teacher, 2.0, 0.4, 0.6)
    out = {k: torch.full_like(v, 7.0) for k, v in want.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(out[k], want[k]) for k in out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (11, 12, 13):
        nx, nw, nb, nl, nt = make(seed)
        for t, v in ((x, nx), (w, nw), (b, nb), (labels, nl), (teacher[0], nt[0]), (teacher[1], nt[1])):
            t.copy_(v)
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = run(torch, B, "bf16", x, w, b, labels, teacher, 2.0, 0.4, 0.6)
        assert all(torch.equal(out[k], want[k]) for k in out)


def test_refusals(torch, B):
    with pytest.raises(ValueError):
        B.ClassLoss(4, 8, 5, torch.float16)
    with pytest.raises(B.BglError):
        B.ClassLoss(4, 8, 5, top=2, temperature=0.0)
    head, x, w = B.ClassLoss(4, 8, 5, top=2), torch.zeros((4, 8), device="cuda"), torch.zeros((5, 8), device="cuda")
    labels, classes, scores = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    good = dict(x=x, weight=w, labels=labels, teacher=(classes, scores))
    for change in (dict(x=torch.zeros((5, 8), device="cuda")), dict(x=x.bfloat16()), dict(x=x.cpu()), dict(weight=torch.zeros((6, 8), device="cuda")),
                   dict(weight=torch.zeros((8, 5), device="cuda").t()), dict(bias=torch.zeros(4, device="cuda")), dict(labels=labels.long()), dict(labels=labels[:3]),
                   dict(teacher=(classes.long(), scores)), dict(teacher=(classes, scores.double())), dict(teacher=(classes[:, :1], scores)),
                   dict(loss=torch.zeros(5, device="cuda")), dict(saved=torch.zeros((4, 2), device="cuda")), dict(weight=w.clone().requires_grad_())):
        with pytest.raises(ValueError):
            head.forward(**{**good, **change})
    head.forward(**good)
    with pytest.raises(B.BglError):
        head.forward(x, w)
    with pytest.raises(B.BglError):
        head.backward(x, w, torch.zeros((4, head.saved_width), device="cuda"), labels=labels)
