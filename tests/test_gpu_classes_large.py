"""Losses over class scores at sizes that are laid out for large tiles, against the definition in 64 bits.

The bounds are those of the small sizes (test_gpu_classes.py: u = 2^-24, a score is off by (D + 4) u (sum|x||w| + |b|)) and what the laid out operands add.
fp32 scores: a value is two halves of a power of two of its row, 2^-22 of itself or 2^-40 of the row's largest off; of two values' product the three larger ones of four
parts are taken: 3 x 2^-22 = 12 u of the product, so D + 16 for D + 4, which 12 columns of zeros give the reference; a value below 2^-18 of its row's largest is off by less
than 2^-40 of that, (x, w)'s product by 2^-40 (|w| max|x| + |x| max|w|), which `far` adds where rows reach so far.
fp32 products: of three bf16 parts each all but the last ones: 4 u, in the 8 u of the bounds.
bf16: products are exact; dz has eleven bits and not eight, so the type's bounds hold for it; below 2^-28 of s + s' it loses bits and is 2^-40 (s + s') off at most, which
`far` adds too."""
import pytest

from test_gpu_classes import B, Reference, V, check, dtype_of, inputs, run, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def check_large(torch, B, kind, data, t=1.0, s=0.3, st=0.7, head=None, far=False):
    x, w, b, labels, teacher = data
    pad = lambda v: torch.cat([v, torch.zeros((len(v), 12), dtype=v.dtype, device="cuda")], 1)      # noqa: E731
    live = None if labels is None else ((labels >= 0) & (labels < len(w)))
    x_ref = x if live is None or teacher is not None else torch.where(live[:, None], x, torch.zeros_like(x))      # (rows without a label may hold anything)
    ref = Reference(torch, pad(x_ref), pad(w), b, labels, teacher, t, V[kind])
    got = run(torch, B, kind, x, w, b, labels, teacher, t, s, st, head=head)
    if labels is not None:
        check("loss", got["loss"], ref.loss, ref.loss_bound)
    if teacher is not None:
        check("teacher_loss", got["teacher_loss"], ref.teacher_loss, ref.teacher_bound)
    want = ref.gradients(s if labels is not None else 0.0, st if teacher is not None else 0.0)
    D = x.shape[1]
    more = [0.0, 0.0, 0.0]
    if far:
        least = 2.0 ** -40 * (abs(s) + t * abs(st))
        more = [least * w.double().abs().sum(0), least * x_ref.double().abs().sum(0), least * len(x)]
    for name, (value, bound), extra in zip(("dx", "dweight", "dbias"), want, more):
        if name != "dbias":
            value, bound = value[:, :D], bound[:, :D]
        check(name, got[name], value, bound + extra)
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [(20_500, 16, 7_100, 3), (8_300, 17, 17_300, 0), (17_000, 9, 16_500, 2)])
def test_pieces(torch, B, kind, n, D, C, k):
    """dz in pieces of rows, of classes, and of both."""
    data = inputs(torch, kind, n, D, C, k, seed=n)
    got = check_large(torch, B, kind, data, t=2.0, s=1.0 / n, st=1.0 / n if k else 0.0)
    for name in ("dx", "dweight"):
        half = run(torch, B, kind, *data, 2.0, 1.0 / n, 1.0 / n if k else 0.0, want=(name,))
        assert torch.equal(half[name], got[name])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [(97, 513, 41_003, 0), (129, 1_021, 15_999, 5), (2_003, 1_001, 1_005, 1), (16_500, 1_000, 129, 0), (40_001, 399, 131, 3), (2_100, 992, 1_024, 2)])
def test_odd_sizes(torch, B, kind, n, D, C, k):
    data = inputs(torch, kind, n, D, C, k, seed=n, pad=5 if n % 2 else 0, bias=n % 3 > 0)
    got = check_large(torch, B, kind, data, t=1.5, s=1.0 / n, st=0.5 / n if k else 0.0)
    again = run(torch, B, kind, *data, 1.5, 1.0 / n, 0.5 / n if k else 0.0)
    assert all(torch.equal(got[i], again[i]) for i in got if got[i] is not None)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_of_other_alignments(torch, B, kind):
    """The operands one value behind a boundary of 16 bytes, and rows of x of an odd stride, beside aligned ones."""
    n, D, C = 500, 512, 8_200
    x, w, b, labels, _ = data = inputs(torch, kind, n, D, C, 0, seed=2)
    check_large(torch, B, kind, data, s=1.0 / n)
    near = lambda v: torch.cat([v.new_zeros(1), v.flatten()])[1:].view(v.shape)      # noqa: E731
    check_large(torch, B, kind, (near(x), near(w), near(b), near(labels), None), s=1.0 / n)
    wide = torch.full((n, D + 3), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, :D] = x
    check_large(torch, B, kind, (wide[:, :D], w, b, labels, None), s=1.0 / n)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_that_differ_much(torch, B, kind):
    """Rows of x and of the weight from the smallest to large numbers, columns too, and scores far apart."""
    n, D, C = 700, 320, 9_100
    x, w, b, labels, teacher = inputs(torch, kind, n, D, C, 3, seed=3, scale=9.0)
    t = dtype_of(torch, kind)
    rows = 2.0 ** -(torch.arange(n, device="cuda") % 7 * 12).float()
    x = (x.float() * rows[:, None]).to(t)
    x[5], x[6, 1:] = 0, 0
    w = (w.float() * 2.0 ** -(torch.arange(C, device="cuda") % 5 * 10).float()[:, None]).to(t)
    w[7] = 0
    check_large(torch, B, kind, (x, w, b, labels, teacher), t=2.0, far=True)
    tiny = (x.float() * 2.0 ** -60).to(t)
    check_large(torch, B, kind, (tiny, w, b, labels, teacher), t=2.0, far=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scales(torch, B, kind):
    """The gradients' factors, small and large: powers of two change nothing else."""
    data = inputs(torch, kind, 400, 512, 9_900, 2, seed=8)
    want = run(torch, B, kind, *data, 2.0, 0.25, 0.5)
    for e in (-60, -20, 20, 40):
        got = run(torch, B, kind, *data, 2.0, 0.25 * 2.0 ** e, 0.5 * 2.0 ** e)
        assert all(torch.equal(got[i].float() * 2.0 ** -e, want[i].float()) for i in ("dx", "dweight", "dbias")), e


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_without_a_gradient_and_classes_taken_out(torch, B, kind):
    n, D, C = 600, 352, 9_600
    x, w, b, labels, _ = inputs(torch, kind, n, D, C, 0, seed=5)
    out = torch.zeros(C, dtype=torch.bool, device="cuda")
    out[:400], out[8_000:] = True, True
    b[out] = -float("inf")
    labels[:] = torch.randint(400, 8_000, (n,), device="cuda", dtype=torch.int32)
    off = torch.zeros(n, dtype=torch.bool, device="cuda")
    off[::7], off[128:256] = True, True
    labels[off] = -1
    got = check_large(torch, B, kind, (x, w, b, labels, None), s=1.0 / n)
    assert (got["dweight"][out] == 0).all() and (got["dbias"][out] == 0).all() and (got["dx"][off] == 0).all()
    clean = run(torch, B, kind, x, w, b, labels, None, s=1.0)
    x2 = x.clone()
    x2[off] = float("nan")
    x2[0], x2[7, 3], x2[14] = float("inf"), -float("inf"), torch.finfo(x.dtype).max
    got = run(torch, B, kind, x2, w, b, labels, None, s=1.0)
    for name in ("loss", "dx", "dweight", "dbias"):
        assert torch.equal(got[name], clean[name]), name
    # one that has a label spoils itself, and no other row's loss and dx
    x2[5, 3] = float("inf")
    got = run(torch, B, kind, x2, w, b, labels, None, s=1.0)
    keep = [i for i in range(n) if i != 5]
    assert not got["loss"][5].isfinite() and got["dx"][5].isnan().all()
    assert torch.equal(got["loss"][keep], clean["loss"][keep]) and torch.equal(got["dx"][keep], clean["dx"][keep])


def test_no_row_has_a_label(torch, B):
    for kind in ("f32", "bf16"):
        x, w, b, labels, teacher = inputs(torch, kind, 900, 300, 8_000, 3, seed=6)
        labels.fill_(-1)
        teacher[0].fill_(8_000)
        x[:] = float("nan")
        got = run(torch, B, kind, x, w, b, labels, teacher, 2.0, 1.0, 1.0)
        assert all((got[k] == 0).all() for k in ("loss", "teacher_loss", "dx", "dweight", "dbias"))


def test_one_object_for_large_and_small_calls(torch, B):
    for kind, D, C in (("f32", 130, 5_100), ("bf16", 200, 17_000)):
        head = B.ClassLoss(9_000, D, C, dtype_of(torch, kind), top=2, temperature=2.0)
        for n in (9_000, 1, 4_095, 100, 600, 0, 8_191):
            data = inputs(torch, kind, n, D, C, 2, seed=n)
            got, want = (run(torch, B, kind, *data, 2.0, 0.1, 0.1, head=h) for h in (head, None))
            assert all(torch.equal(got[i], want[i]) for i in got), n


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_two_graphs_and_eager_calls(torch, B, kind):
    """Two captured calls of one object, replayed in turn between eager ones of another."""
    n, D, C = 600, 384, 9_300
    make = lambda seed: inputs(torch, kind, n, D, C, 4, seed=seed)      # noqa: E731
    head = B.ClassLoss(n, D, C, dtype_of(torch, kind), top=4, temperature=2.0)
    calls = []
    for seed in (1, 2):
        x, w, b, labels, teacher = data = make(seed)
        out = {k: torch.full_like(v, 7.0) for k, v in run(torch, B, kind, *data, 2.0, 0.4, 0.6).items()}
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            head.forward(x, w, bias=b, labels=labels, teacher=teacher, loss=out["loss"], teacher_loss=out["teacher_loss"], saved=out["saved"])
            head.backward(x, w, out["saved"], bias=b, labels=labels, teacher=teacher, scale=0.4, teacher_scale=0.6, dx=out["dx"], dweight=out["dweight"], dbias=out["dbias"])
        calls.append((data, out, graph))
    for seed in (11, 12, 13):
        for i, (data, out, graph) in enumerate(calls):
            nx, nw, nb, nl, nt = make(seed + 20 * i)
            for t, v in zip((*data[:4], *data[4]), (nx, nw, nb, nl, *nt)):
                t.copy_(v)
            for t in out.values():
                t.fill_(float("nan"))
            graph.replay()
            want = run(torch, B, kind, *data, 2.0, 0.4, 0.6)
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in out), (seed, i)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 128])
def test_a_weight_beyond_32_bits(torch, B, kind, n):
    """Classes from 2^31 values of the weight on; all others are taken out, so that the call of these alone is the same one."""
    D, C, far = 260, 2_000, 8_300_000
    x, w, b, labels, teacher = inputs(torch, kind, n, D, C, 3, seed=9)
    small = run(torch, B, kind, x, w, b, labels, teacher, 2.0, 0.5, 0.5)
    ref = Reference(torch, torch.cat([x, x.new_zeros((n, 12))], 1), torch.cat([w, w.new_zeros((C, 12))], 1), b, labels, teacher, 2.0, V[kind])
    assert far * D > 2 ** 31
    ref.sum += far / 1000 * 2.0 ** -24      # (more parts of a sum, those of the others 0)
    w_all, b_all = torch.zeros((far + C, D), dtype=w.dtype, device="cuda"), torch.full((far + C,), -float("inf"), dtype=b.dtype, device="cuda")
    w_all[far:], b_all[far:] = w, b
    place = lambda c: torch.where((c >= 0) & (c < C), c + far, -1).int()      # noqa: E731
    got = run(torch, B, kind, x, w_all, b_all, place(labels), (place(teacher[0]), teacher[1]), 2.0, 0.5, 0.5)
    more = far / 1000 * 2.0 ** -24
    check("loss", got["loss"], ref.loss, ref.loss_bound + more)
    check("teacher_loss", got["teacher_loss"], ref.teacher_loss, ref.teacher_bound + 4 * more)
    assert (got["dweight"][:far] == 0).all() and (got["dbias"][:far] == 0).all()
    # both calls' gradients are within the bound of the value, with q off by what the sum is
    for name, value, (want, bound) in zip(("dx", "dweight", "dbias"), (got["dx"], got["dweight"][far:], got["dbias"][far:]), ref.gradients(0.5, 0.5)):
        want, bound = (want, bound) if name == "dbias" else (want[:, :D], bound[:, :D])
        check(name, small[name], want, bound)
        size = {"dx": w.double().abs().sum(0), "dweight": x.double().abs().sum(0), "dbias": n}[name]
        check(name, value, want, bound + 2 * more * size)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("C", [7, 150])
def test_rows_beyond_32_bits(torch, B, kind, C):
    """The same rows 2,100 times: the same losses and dx each time; labels in the last ones alone: their dweight."""
    n, D, times = 8_192, 130, 2_100
    x, w, b, labels, _ = inputs(torch, kind, n, D, C, 0, seed=10)
    head = B.ClassLoss(n * times, D, C, dtype_of(torch, kind))
    all_x, saved = x.repeat(times, 1), torch.full((n * times, 2), 7.0, device="cuda")
    assert all_x.numel() > 2 ** 31
    loss, dx = torch.full((n * times,), 7.0, device="cuda"), torch.full_like(all_x, 7.0)
    head.forward(all_x, w, bias=b, labels=labels.repeat(times), loss=loss, saved=saved)
    head.backward(all_x, w, saved, bias=b, labels=labels.repeat(times), dx=dx)
    ref = Reference(torch, torch.cat([x, x.new_zeros((n, 12))], 1), torch.cat([w, w.new_zeros((C, 12))], 1), b, labels, None, 1.0, V[kind])
    check("loss", loss[-n:], ref.loss, ref.loss_bound)
    (want_dx, dx_bound), (want_dw, dw_bound), (want_db, db_bound) = ref.gradients(1.0, 0.0)
    check("dx", dx[-n:], want_dx[:, :D], dx_bound[:, :D])
    assert (loss.view(times, n) == loss[-n:]).all()
    for part in dx.view(times, n, D).split(100):
        assert (part == dx[-n:]).all()
    some = torch.full((n * times,), -1, dtype=torch.int32, device="cuda")
    some[-n:] = labels
    dw, db = torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    head.backward(all_x, w, saved, bias=b, labels=some, dweight=dw, dbias=db)
    check("dweight", dw, want_dw[:, :D], dw_bound[:, :D])
    check("dbias", db, want_db, db_bound)


def test_another_device_is_refused(torch, B):
    """An object made on another device than the current one, as far as one device can show it."""
    x, w, labels = torch.zeros((4, 8), device="cuda"), torch.zeros((5, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for make, call in ((lambda: B.ClassLoss(4, 8, 5), lambda o: o.forward(x, w, labels=labels)), (lambda: B.ClassLoss(4, 8, 5), lambda o: o.backward(x, w, torch.zeros((4, 2), device="cuda"), labels=labels, dx=x)),
                       (lambda: B.LayerNorm(4, 8), lambda o: o.forward(x, x)), (lambda: B.LayerNorm(4, 8), lambda o: o.backward(x, x, torch.zeros((4, 2), device="cuda"), dx=x))):
        o = make()
        o._device += 1
        with pytest.raises(ValueError, match="device"):
            call(o)
    with pytest.raises(ValueError, match="device"):
        B.LayerNorm(4, 8).forward(x, x.cpu())


@pytest.mark.parametrize("t", [1.0, 2.0])
def test_gradients_near_certainty(torch, B, t):
    """Scores that are exact, up to 60 and within 4 of each other, and the weight of the identity, so that dx is dz: right to 16 u of 1 however large the scores are.  A
    power is off by 2 u and by what its argument is, half a step of one below 8 over log2(e): 4 u; a sum of two by as much; their quotient and the rest by 4 roundings:
    together 2 (2 + 4) + 4 = 16 u."""
    n, u = 400, 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(1)
    high = torch.randint(40, 240, (n,), generator=g, device="cuda") / 4
    x = torch.stack([high, high - torch.randint(0, 17, (n,), generator=g, device="cuda") / 4], 1)
    x[::2] = x[::2].flip(1)
    w = torch.eye(2, device="cuda")
    labels = torch.randint(0, 2, (n,), generator=g, device="cuda", dtype=torch.int32)
    z, onehot = x.double(), torch.nn.functional.one_hot(labels.long(), 2).double()
    got = run(torch, B, "f32", x, w, None, labels, None, s=1.0, want=("dx", "dweight"))
    assert ((got["dx"].double() - (z.softmax(1) - onehot)).abs() <= 16 * u).all()
    classes = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").repeat(n, 1)
    classes[::3] = classes[::3].flip(1)
    classes[5], classes[7, 0] = 1, -1
    scores = torch.randint(-8, 8, (n, 2), generator=g, device="cuda") / 4
    e = (scores.double() / t).exp() * (classes >= 0)
    p = torch.zeros((n, 2), dtype=torch.float64, device="cuda").scatter_add_(1, classes.clamp_min(0).long(), e / e.sum(1, keepdim=True))
    got = run(torch, B, "f32", x, w, None, None, (classes, scores), t, 0.0, 1.0, want=("dx", "dweight"))
    # (the teacher's p as well, its arguments below 8 too; the factor t is exact)
    assert ((got["dx"].double() - t * ((z / t).softmax(1) - p)).abs() <= 2 * 16 * u * t).all()
