"""Layer norm and its gradients against the definition in 64 bits.

u = 2^-24 is the unit roundoff of the sums, v that of the type (2^-24 or 2^-8).  A row's sums are added in at most 16 + 10 + 2 steps (a thread's
values, the lanes and wavefronts of a team), so that a sum of exact terms is off by less than 30 u of the terms' absolute sum.  The mean is first m, then
corrected by the mean of the rounded x - m, and kept in fp32: off by 30 u mean|x - mean| + u |mean|.  Squares' sum 34 u, so r 18 u with its root and
quotient.  h = (x - mean) r is therefore off by H = 20 u |h| + 30 u + u |mean| r (r mean|x - mean| <= 1).  What follows is linear in these."""
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
    def __init__(self, x, w, b, eps, v):
        n, width = x.shape
        self.x, self.v, self.width = x, v, width
        self.g = np.ones(width) if w is None else w
        bias = np.zeros(width) if b is None else b
        mean = x.mean(1, keepdims=True)
        self.r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
        self.h = (x - mean) * self.r
        self.H = 20 * U * np.abs(self.h) + 30 * U + U * np.abs(mean) * self.r
        self.y = self.h * self.g + bias
        self.y_bound = np.abs(self.g) * self.H + 2 * U * (np.abs(self.h * self.g) + np.abs(bias)) + 1.01 * v * np.abs(self.y) + 1e-37

    def gradients(self, dy):
        d, h, H, r = dy * self.g, self.h, self.H, self.r
        c1, c2 = d.mean(1, keepdims=True), (d * h).mean(1, keepdims=True)
        e1 = 32 * U * np.abs(d).mean(1, keepdims=True)
        e2 = 34 * U * np.abs(d * h).mean(1, keepdims=True) + (np.abs(d) * H).mean(1, keepdims=True)
        dx = r * (d - c1 - h * c2)
        bound = r * (24 * U * (np.abs(d) + np.abs(c1) + np.abs(h * c2)) + e1 + np.abs(h) * e2 + H * (np.abs(c2) + e2)) + 1.01 * self.v * np.abs(dx) + 1e-37
        # over rows: a thread's, its workgroup's teams (up to 32), the partial rows' eighths (up to 128) and these (8)
        steps = min(len(dy), len(dy) / 1024 + 1 + 32 + 128 + 8) + 4
        dw, db = (dy * h).sum(0), dy.sum(0)
        dwb = steps * U * np.abs(dy * h).sum(0) + (np.abs(dy) * H).sum(0) + 1.01 * self.v * np.abs(dw) + 1e-37
        dbb = steps * U * np.abs(dy).sum(0) + 1.01 * self.v * np.abs(db) + 1e-37
        return (dx, bound), (dw, dwb), (db, dbb)


def check(name, got, want, bound):
    got = got.double().cpu().numpy()
    over = np.abs(got - want) - bound
    assert np.isfinite(got).all(), name
    assert (over <= 0).all(), f"{name}: {np.abs(got - want).max()} off, worst {over.max()} beyond its bound at {np.unravel_index(over.argmax(), over.shape)}"


def inputs(torch, kind, n, width, seed, shift=0.0, spread=1.0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = dtype_of(torch, kind)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    rows = lambda a: a.to(t) if not pad else torch.cat([a.to(t), torch.full((n, pad), float("nan"), dtype=t, device="cuda")], 1)[:, :width]      # noqa: E731
    x = rows(rnd(n, width) * spread * torch.exp(rnd(n, 1)) + shift * rnd(n, 1))
    return x, (1 + 0.3 * rnd(width)).to(t), (0.5 * rnd(width)).to(t), rows(rnd(n, width))


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def run_both(torch, B, kind, x, w, b, dy, eps=1e-5, want=("dx", "dweight", "dbias"), stream=None):
    n, width = x.shape
    t = dtype_of(torch, kind)
    norm = B.LayerNorm(n, width, t, eps)
    out = dict(y=torch.full((n, width), 7.0, dtype=t, device="cuda"), saved=torch.empty((n, 2), device="cuda"), dx=torch.full((n, width), 7.0, dtype=t, device="cuda"),
               dweight=torch.full((width,), 7.0, dtype=t, device="cuda"), dbias=torch.full((width,), 7.0, dtype=t, device="cuda"))
    norm.forward(x, out["y"], weight=w, bias=b, saved=out["saved"], stream=stream)
    norm.backward(dy, x, out["saved"], weight=w, stream=stream, **{k: out[k] for k in want})
    return out


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 100, 127, 128, 129, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2050, 4096, 5001, 8192, 8193, 16384]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_every_width(torch, B, kind, width):
    for n, affine, pad in [(1, True, 0), (37, True, 0), (70, False, 3)]:
        x, w, b, dy = inputs(torch, kind, n, width, seed=width * 10 + n, shift=1.0, pad=pad)
        if not affine:
            w = b = None
        ref = Reference(np64(x), np64(w), np64(b), 1e-5, V[kind])
        got = run_both(torch, B, kind, x, w, b, dy)
        what = f"width {width}, {n} rows"
        check(f"y, {what}", got["y"], ref.y, ref.y_bound)
        for name, (value, bound) in zip(("dx", "dweight", "dbias"), ref.gradients(np64(dy))):
            check(f"{name}, {what}", got[name], value, bound)


@pytest.mark.parametrize("kind,n,width", [("f32", 40_000, 100), ("bf16", 40_000, 136), ("f32", 20_011, 33), ("bf16", 5_000, 1_100), ("f32", 2_500, 2_100)])
def test_many_rows(torch, B, kind, n, width):
    x, w, b, dy = inputs(torch, kind, n, width, seed=n)
    ref = Reference(np64(x), np64(w), np64(b), 1e-5, V[kind])
    got = run_both(torch, B, kind, x, w, b, dy)
    check("y", got["y"], ref.y, ref.y_bound)
    for name, (value, bound) in zip(("dx", "dweight", "dbias"), ref.gradients(np64(dy))):
        check(name, got[name], value, bound)
    again = run_both(torch, B, kind, x, w, b, dy)
    assert all(torch.equal(got[k], again[k]) for k in got)
    half = run_both(torch, B, kind, x, w, b, dy, want=("dx",))
    assert torch.equal(half["dx"], got["dx"]) and (half["dweight"] == 7).all() and (half["dbias"] == 7).all()
    sums = run_both(torch, B, kind, x, w, b, dy, want=("dweight",))
    assert torch.equal(sums["dweight"], got["dweight"]) and (sums["dx"] == 7).all() and (sums["dbias"] == 7).all()


@pytest.mark.parametrize("width", [5, 100, 1_500])
@pytest.mark.parametrize("shift,spread,eps", [(1e4, 1.0, 1e-5), (0.0, 1e-6, 1e-12), (0.0, 1e22, 1e-5), (1e30, 1e35, 1e-5), (1.0, 0.0, 1e-5)])
def test_rows_far_from_zero_tiny_and_huge(torch, B, width, shift, spread, eps):
    x, w, b, dy = inputs(torch, "f32", 19, width, seed=3, shift=shift, spread=spread)
    ref = Reference(np64(x), np64(w), np64(b), eps, V["f32"])
    got = run_both(torch, B, "f32", x, w, b, dy, eps)
    check("y", got["y"], ref.y, ref.y_bound)
    for name, (value, bound) in zip(("dx", "dweight", "dbias"), ref.gradients(np64(dy))):
        check(name, got[name], value, bound + 2.0 ** -140)       # (gradients of huge rows are near the smallest numbers)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", [24, 700, 3_000])
def test_a_row_that_is_not_finite_stays_alone(torch, B, kind, width):
    x, w, b, dy = inputs(torch, kind, 12, width, seed=5)
    clean = run_both(torch, B, kind, x, w, b, dy)
    x2 = x.clone()
    x2[3, width // 2], x2[7, 0], x2[11, width - 1] = float("nan"), float("inf"), float("-inf")
    got = run_both(torch, B, kind, x2, w, b, dy)
    keep = [i for i in range(12) if i not in (3, 7, 11)]
    for k in ("y", "dx"):
        assert torch.equal(got[k][keep], clean[k][keep])
        assert got[k][[3, 7, 11]].isnan().all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_in_place_and_beside_other_values(torch, B, kind):
    t = dtype_of(torch, kind)
    for width in (36, 130, 2_000):
        x, w, b, dy = inputs(torch, kind, 50, width, seed=8)
        want = run_both(torch, B, kind, x, w, b, dy)
        room = torch.full((52, width + 5), 3.0, dtype=t, device="cuda")
        xs, norm = room[1:51, 2:2 + width], B.LayerNorm(60, width, t)
        xs.copy_(x)
        saved = torch.empty((50, 2), device="cuda")
        norm.forward(xs, xs, weight=w, bias=b, saved=saved)
        assert torch.equal(xs, want["y"]) and torch.equal(saved, want["saved"])
        xs.copy_(dy)
        norm.backward(xs, x, saved, weight=w, dx=xs)
        assert torch.equal(xs, want["dx"])
        xs.fill_(3.0)
        assert (room == 3).all()


def test_gradients_are_differences(torch, B):
    x, w, b, dy = inputs(torch, "f32", 6, 11, seed=4)
    got = run_both(torch, B, "f32", x, w, b, dy)
    X, W, Bi, D = np64(x), np64(w), np64(b), np64(dy)
    loss = lambda x, w, b: (Reference(x, w, b, 1e-5, 0).y * D).sum()      # noqa: E731
    step = 1e-5
    for name, at, of in (("dx", 0, X), ("dweight", 1, W), ("dbias", 2, Bi)):
        grad = np.empty_like(of)
        for i in np.ndindex(of.shape):
            args = [X.copy(), W.copy(), Bi.copy()]
            args[at][i] += step
            up = loss(*args)
            args[at][i] -= 2 * step
            grad[i] = (up - loss(*args)) / (2 * step)
        # central differences: third derivatives times step^2 (1e-10 x some hundreds), rounding 1e-16 x 1e2 / 1e-5; the kernel 1e-5
        np.testing.assert_allclose(np64(got[name]), grad, atol=2e-5, rtol=2e-5)


def test_no_rows(torch, B):
    norm = B.LayerNorm(10, 20)
    e, s = torch.empty((0, 20), device="cuda"), torch.empty((0, 2), device="cuda")
    dw, db = torch.full((20,), 7.0, device="cuda"), torch.full((20,), 7.0, device="cuda")
    norm.forward(e, e, saved=s)
    norm.backward(e, e, s, dx=e, dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


def test_offsets_beyond_32_bits(torch, B):
    n, stride, width = 1_100, 1 << 21, 64
    room = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    x, w, b, dy = inputs(torch, "bf16", n, width, seed=9)
    far = room.view(n, stride)[:, :width]
    far.copy_(x)
    want, norm = run_both(torch, B, "bf16", x, w, b, dy), B.LayerNorm(n, width, torch.bfloat16)
    saved, dx = torch.empty((n, 2), device="cuda"), torch.empty_like(x)
    norm.forward(far, far, weight=w, bias=b, saved=saved)
    assert torch.equal(far, want["y"])
    far.copy_(x)
    norm.backward(dy, far, saved, weight=w, dx=dx)
    assert torch.equal(dx, want["dx"])


def test_graph_and_other_stream(torch, B):
    x, w, b, dy = inputs(torch, "bf16", 900, 300, seed=6)
    norm = B.LayerNorm(900, 300, torch.bfloat16)
    y, dx, dw, db, saved = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b), torch.empty((900, 2), device="cuda")

    def both(stream=None):
        norm.forward(x, y, weight=w, bias=b, saved=saved, stream=stream)
        norm.backward(dy, x, saved, weight=w, dx=dx, dweight=dw, dbias=db, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.current_stream().wait_stream(side)
    want = run_both(torch, B, "bf16", x, w, b, dy)
    assert all(torch.equal(a, want[k]) for a, k in ((y, "y"), (dx, "dx"), (dw, "dweight"), (db, "dbias")))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (11, 12, 13):
        nx, _, _, ndy = inputs(torch, "bf16", 900, 300, seed=seed)
        x.copy_(nx), dy.copy_(ndy)
        for t in (y, dx, dw, db, saved):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = run_both(torch, B, "bf16", x, w, b, dy)
        assert all(torch.equal(a, want[k]) for a, k in ((y, "y"), (dx, "dx"), (dw, "dweight"), (db, "dbias")))


def test_refusals(torch, B):
    with pytest.raises(ValueError):
        B.LayerNorm(4, 8, torch.float16)
    with pytest.raises(B.BglError):
        B.LayerNorm(4, 8, eps=0.0)
    norm, x = B.LayerNorm(4, 8), torch.zeros((4, 8), device="cuda")
    saved = torch.empty((4, 2), device="cuda")
    bad = [dict(x=torch.zeros((5, 8), device="cuda"), y=torch.zeros((5, 8), device="cuda")), dict(x=x, y=torch.zeros((4, 9), device="cuda")),
           dict(x=x.bfloat16(), y=x), dict(x=x.cpu(), y=x), dict(x=x, y=x, weight=torch.zeros(9, device="cuda")), dict(x=x.t().contiguous().t(), y=x),
           dict(x=x, y=x, saved=torch.empty((4, 3), device="cuda")), dict(x=x, y=x, saved=saved.double()), dict(x=x.clone().requires_grad_(), y=x)]
    for call in bad:
        with pytest.raises(ValueError):
            norm.forward(**call)
    with torch.no_grad():
        norm.forward(x.clone().requires_grad_(), x)
    with pytest.raises(B.BglError):
        norm.backward(x, x, None, dx=x)
