"""Layers over a batch's rows, layers by group, and the grouping, against plain loops over the definition in 64 bits.

The bounds are error bounds of the arithmetic, element by element.  u = 2^-24 (fp32) is the unit roundoff of the sums, v that of the
type (2^-24 or 2^-8).  A sum of K products of exact factors in any order is off by at most (K + 2) u sum|.||.|; z adds the bias and the residual.
An activation with slope at most 1.13 passes that on and adds its own evaluation (32 u (1 + |z|)).  dz sees z rounded to the type
(second derivatives are at most 0.8), is itself rounded to the type, and each of its errors is then multiplied out in dx, dW and db."""
import itertools

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ACTS = ["none", "relu", "gelu", "silu"]


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


def act64(name, z):
    from scipy.special import erf
    with np.errstate(over="ignore"):
        if name == "relu":
            return np.maximum(z, 0), (z > 0).astype(np.float64)
        if name == "gelu":
            p = 0.5 * (1 + erf(z / np.sqrt(2)))
            return z * p, p + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        if name == "silu":
            p = 1 / (1 + np.exp(-z))
            return z * p, p * (1 + z * (1 - p))
    return z, np.ones_like(z)


class Reference:
    """The layer in 64 bits with a bound beside each value.  group: of each row (-1: none), or None."""

    def __init__(self, x, w, b, r, mode, act, v, group=None):
        self.x, self.w, self.act, self.v = x, w, act, v
        self.G = w.shape[0]
        n, K = x.shape
        self.members = [np.arange(n)] if group is None else [np.nonzero(group == g)[0] for g in range(self.G)]
        N = w.shape[1]
        z, bound = np.zeros((n, N)), np.zeros((n, N))
        for g, at in enumerate(self.members):
            z[at] = x[at] @ w[g].T + (0 if b is None else b[g])
            bound[at] = (K + 4) * U * (np.abs(x[at]) @ np.abs(w[g]).T + (0 if b is None else np.abs(b[g])))
        if mode == "before":
            z, bound = z + r, bound + (K + 4) * U * np.abs(r)
        self.z, self.z_bound = z, bound
        self.y, self.slope = act64(act, z)
        self.y_bound = 1.13 * bound + (32 * U * (1 + np.abs(z)) if act in ("gelu", "silu") else 0)
        if mode == "after":
            self.y, self.y_bound = self.y + r, self.y_bound + 2 * U * (np.abs(self.y) + np.abs(r))
        self.y_bound = self.y_bound + v * np.abs(self.y) * 1.01 + 1e-30

    def gradients(self, dy, want_bias):
        v = self.v
        dz = dy * self.slope
        dzb = np.abs(dy) * (0.8 * (self.z_bound + v * np.abs(self.z)) + 32 * U * (1 + np.abs(self.z))) + v * np.abs(dz) * 1.01
        if self.act == "none":
            dzb = np.zeros_like(dz)                  # dz is dy
        if self.act == "relu":                       # slope 0 or 1: off only where the sign may be
            dzb = np.where(np.abs(self.z) <= self.z_bound, np.abs(dy), 0)
        n, K = self.x.shape
        N = self.w.shape[1]
        dx, dxb = np.zeros((n, K)), np.zeros((n, K))
        dw, dwb, db, dbb = (np.zeros(s) for s in (self.w.shape, self.w.shape, (self.G, N), (self.G, N)))
        for g, at in enumerate(self.members):
            d, e, ax, aw = dz[at], dzb[at], np.abs(self.x[at]), np.abs(self.w[g])
            dx[at] = d @ self.w[g]
            dxb[at] = e @ aw + (N + 4) * U * ((np.abs(d) + e) @ aw)
            dw[g] = d.T @ self.x[at]
            dwb[g] = e.T @ ax + (len(at) + 4) * U * ((np.abs(d) + e).T @ ax)
            db[g] = d.sum(0)
            dbb[g] = e.sum(0) + (len(at) + 4) * U * (np.abs(d) + e).sum(0)
        out = dict(dx=(dx, dxb), dweight=(dw, dwb), dresidual=(dz, dzb), dbias=(db, dbb))
        return {k: (a, e + v * np.abs(a) * 1.01 + 1e-30) for k, (a, e) in out.items()}


def close(name, got, want, bound):
    got = got.double().cpu().numpy().reshape(want.shape)
    off = np.abs(got - want)
    assert np.isfinite(got).all(), f"{name}: not finite"
    worst = np.max(off / bound) if off.size else 0.0
    assert worst <= 1.0, f"{name}: {worst:.2f} times the bound"


def rows_of(torch, rng, n, width, dtype, pad=0, shift=0):
    """n rows on the GPU, `pad` values apart, the first `shift` values into its memory; (view, values in 64 bits)."""
    t = torch.full((n * (width + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    view = t[shift: shift + n * (width + pad)].view(n, width + pad)[:, :width]
    view.copy_(torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)).to(dtype))
    return view, view.double().cpu().numpy()


def run_layer(torch, B, dtype, n, K, N, act, mode, bias=True, groups=0, pad=0, shift=0, seed=0, stream=None):
    dt = dtype_of(torch, dtype)
    rng = np.random.default_rng([seed, n, K, N])
    G = max(groups, 1)
    x, x64 = rows_of(torch, rng, n, K, dt, pad, shift)
    w = torch.from_numpy((rng.standard_normal((G, N, K)) / np.sqrt(K)).astype(np.float32)).to(dt).cuda()
    b = torch.from_numpy(rng.standard_normal((G, N)).astype(np.float32)).to(dt).cuda() if bias else None
    r, r64 = rows_of(torch, rng, n, N, dt, pad, shift) if mode != "none" else (None, None)
    dy, dy64 = rows_of(torch, rng, n, N, dt, pad, shift)
    group, rg = None, None
    if groups:
        group = rng.integers(-1, groups, n).astype(np.int32)
        if groups > 2:
            group[group == groups - 2] = groups // 2 - 1            # a group without rows
        rg = B.RowGroups(n, groups)
        rg.build(torch.from_numpy(group).cuda())
    ref = Reference(x64, w.double().cpu().numpy(), None if b is None else b.double().cpu().numpy(), r64, mode, act,
                    U if dtype == "f32" else 2.0 ** -8, group)
    lay = B.Linear(n, K, N, dt, act, mode, groups)
    y, _ = rows_of(torch, rng, n, N, dt, pad, shift)
    dx, _ = rows_of(torch, rng, n, K, dt, pad, shift)
    saved = rows_of(torch, rng, n, N, dt, pad, shift)[0] if act != "none" else None
    dres = rows_of(torch, rng, n, N, dt, pad, shift)[0] if mode == "before" else None
    dw, db = torch.full_like(w, float("nan")), torch.full_like(b, float("nan")) if bias else None
    one = lambda t: t if t is None or groups else t[0]      # noqa: E731
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    lay.forward(x, one(w), y, one(b), r, saved, rg, stream)
    lay.backward(dy, x, one(w), saved, dx, one(dw), one(db), dres, rg, stream)
    torch.cuda.synchronize()
    close("y", y, ref.y, ref.y_bound)
    want = ref.gradients(dy64, bias)
    close("dx", dx, *want["dx"])
    close("dweight", dw, *want["dweight"])
    if bias:
        close("dbias", db, *want["dbias"])
    if dres is not None:
        close("dresidual", dres, *want["dresidual"])
    if pad:      # what lies between the rows is nobody's
        for t in (y, dx):
            assert bool(torch.isnan(torch.as_strided(t, (t.shape[0] - 1, pad), t.stride(), t.storage_offset() + t.shape[1])).all())


SIZES = [(1, 1, 1), (1, 512, 512), (2, 31, 64), (3, 7, 5), (16, 256, 100), (17, 64, 65), (64, 64, 64), (65, 33, 129), (127, 100, 47),
         (130, 257, 70), (300, 129, 130), (1000, 100, 128), (5485, 100, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,N", SIZES)
def test_layer_matches_the_definition(torch, B, dtype, n, K, N):
    i = SIZES.index((n, K, N))
    run_layer(torch, B, dtype, n, K, N, ACTS[i % 4], ["none", "before", "after"][i % 3])
    run_layer(torch, B, dtype, n, K, N, ACTS[(i + 2) % 4], ["before", "after", "none"][i % 3], bias=False)


@pytest.mark.parametrize("dtype,act,mode", itertools.product(["f32", "bf16"], ACTS, ["none", "before", "after"]))
def test_every_epilogue(torch, B, dtype, act, mode):
    run_layer(torch, B, dtype, 150, 40, 72, act, mode, seed=1)
    run_layer(torch, B, dtype, 150, 40, 72, act, mode, groups=3, seed=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 2), (8, 0), (5, 7)])
def test_strides_and_alignment(torch, B, dtype, pad, shift):
    run_layer(torch, B, dtype, 90, 64, 96, "silu", "before", pad=pad, shift=shift, seed=2)
    run_layer(torch, B, dtype, 90, 45, 33, "gelu", "after", pad=pad, shift=shift, groups=4, seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_in_the_large_tiles(torch, B, dtype):
    run_layer(torch, B, dtype, 33_001, 40, 100, "gelu", "none", seed=4)
    run_layer(torch, B, dtype, 33_001, 100, 72, "none", "after", groups=5, seed=5)
    run_layer(torch, B, dtype, 17_000, 130, 257, "relu" if dtype == "bf16" else "silu", "before", seed=6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,N,G", [(1, 16, 16, 2), (5, 100, 64, 70), (37, 256, 256, 8), (64, 8, 8, 64), (777, 50, 30, 130),
                                     (2049, 100, 64, 4), (6000, 64, 128, 3), (3000, 12, 20, 1024)])
def test_grouped_layer_matches_the_definition(torch, B, dtype, n, K, N, G):
    run_layer(torch, B, dtype, n, K, N, "silu", "before", groups=G, seed=7)
    run_layer(torch, B, dtype, n, K, N, "none", "none", groups=G, seed=8)


@pytest.mark.parametrize("n,G", [(0, 3), (1, 1), (63, 5), (64, 64), (2047, 7), (2048, 1024), (2049, 7), (50_001, 1), (50_000, 24),
                                 (428_377, 1000)])
@pytest.mark.parametrize("with_ids", [False, True])
def test_grouping_is_a_stable_sort(torch, B, n, G, with_ids):
    rng = np.random.default_rng([n, G])
    nodes = 2 * n + 5
    of = rng.integers(-2, G + 2, nodes).astype(np.int32)
    ids = rng.integers(-3, nodes + 3, n).astype(np.int32)       # some outside the table
    g = B.RowGroups(n + 10, G)
    g.build(torch.from_numpy(of).cuda(), torch.from_numpy(ids).cuda() if with_ids else None, n=n)
    key = np.where((ids >= 0) & (ids < nodes), of[np.clip(ids, 0, nodes - 1)], -1) if with_ids else of[:n]
    key = np.where((key >= 0) & (key < G), key, G)
    assert np.array_equal(g.rows.cpu().numpy(), np.argsort(key, kind="stable"))
    assert np.array_equal(g.offsets.cpu().numpy(), np.searchsorted(np.sort(key), np.arange(G + 1)))


def test_groups_of_rows_already_in_order_and_rows_left_out(torch, B):
    """The C call without a row list; with one that names positions outside the batch; with offsets that lead outside."""
    n, K, N, G = 200, 24, 40, 3
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.standard_normal((n, K)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.standard_normal((G, N, K)).astype(np.float32)).cuda()
    st = B.LinearStruct(0, 0, 0, K, N, G)
    x64, w64 = x.double().cpu().numpy(), w.double().cpu().numpy()

    def call(rows, offsets):
        import ctypes as C
        y = torch.full((n, N), -7.0, device="cuda")
        B._check(B.lib().bgl_linear_forward(C.byref(st), n, None if rows is None else rows.data_ptr(), offsets.data_ptr(), x.data_ptr(), K,
                                            w.data_ptr(), None, None, 0, y.data_ptr(), N, None, 0, B._stream_handle(None)))
        return y.cpu().numpy()
    offsets = torch.tensor([0, 70, 70, 150], dtype=torch.int32).cuda()
    want = np.concatenate([x64[:70] @ w64[0].T, x64[70:150] @ w64[2].T, np.zeros((50, N))])
    assert np.allclose(call(None, offsets), want, atol=(K + 4) * U * 60)
    rows = np.arange(n, dtype=np.int32)[::-1].copy()
    rows[[0, 100, 160]] = [-1, n, 2**31 - 1]
    got = call(torch.from_numpy(rows).cuda(), offsets)
    group = np.full(n, 3)
    group[:70], group[70:150] = 0, 2
    named = (rows >= 0) & (rows < n)
    for s in np.nonzero(named)[0]:
        r = rows[s]
        ref = x64[r] @ w64[group[s]].T if group[s] < G else np.zeros(N)
        assert np.allclose(got[r], ref, atol=(K + 4) * U * 60)
    untouched = np.setdiff1d(np.arange(n), rows[named])
    assert len(untouched) == 3 and (got[untouched] == -7.0).all()
    wild = call(None, torch.tensor([0, 1 << 30, -5, 120], dtype=torch.int32).cuda())     # group 0 has all rows, the others overlap it
    assert np.isfinite(wild).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,typed", [(5000, 0), (5000, 1), (5000, 70), (40_000, 130)])
def test_batches_whose_rows_mostly_belong_to_no_group(torch, B, dtype, n, typed):
    """Fewer groups' rows than the backward call planned shares for."""
    dt, K, N, G = dtype_of(torch, dtype), 40, 24, 4
    rng = np.random.default_rng([n, typed])
    group = np.full(n, -1, dtype=np.int32)
    group[rng.permutation(n)[:typed]] = rng.integers(0, G, typed)
    x, x64 = rows_of(torch, rng, n, K, dt)
    dy, dy64 = rows_of(torch, rng, n, N, dt)
    w = torch.from_numpy(rng.standard_normal((G, N, K)).astype(np.float32)).to(dt).cuda()
    ref = Reference(x64, w.double().cpu().numpy(), None, None, "none", "none", U if dtype == "f32" else 2.0 ** -8, group)
    rg, lay = B.RowGroups(n, G), B.Linear(n, K, N, dt, num_groups=G)
    rg.build(torch.from_numpy(group).cuda())
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.full_like(w, float("nan")), torch.full((G, N), float("nan"), dtype=dt, device="cuda")
    lay.workspace = B._workspace(lay._bytes(n)).view(torch.uint8).fill_(0xFF)      # NaN wherever nothing is written
    lay.forward(x, w, y, groups=rg)
    lay.backward(dy, x, w, dx=dx, dweight=dw, dbias=db, groups=rg)
    want = ref.gradients(dy64, True)
    close("y", y, ref.y, ref.y_bound)
    close("dx", dx, *want["dx"])
    close("dweight", dw, *want["dweight"])
    close("dbias", db, *want["dbias"])


def test_no_rows(torch, B):
    for groups in (0, 3):
        lay = B.Linear(0, 8, 5, torch.float32, "relu", "none", groups)
        lead = (groups,) if groups else ()
        w = torch.randn(lead + (5, 8), device="cuda")
        dw, db = torch.full_like(w, 3.0), torch.full(lead + (5,), 3.0, device="cuda")
        e = lambda k: torch.empty((0, k), device="cuda")      # noqa: E731
        rg = None
        if groups:
            rg = B.RowGroups(0, groups)
            rg.build(torch.empty(0, dtype=torch.int32, device="cuda"))
        lay.forward(e(8), w, e(5), saved=e(5), groups=rg)
        lay.backward(e(5), e(8), w, saved=e(5), dx=e(8), dweight=dw, dbias=db, groups=rg)
        torch.cuda.synchronize()
        assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [9, 300])
def test_values_that_are_not_finite_stay_in_their_row(torch, B, dtype, n):
    dt = dtype_of(torch, dtype)
    K, N = 72, 80
    x = torch.ones((n, K), dtype=dt, device="cuda")
    w = torch.ones((N, K), dtype=dt, device="cuda")
    x[1, 3], x[4, 5], x[7, 0] = float("inf"), float("nan"), float("-inf")
    lay = B.Linear(n, K, N, dt)
    y = torch.empty((n, N), dtype=dt, device="cuda")
    lay.forward(x, w, y)
    got = y.float().cpu().numpy()
    assert np.isposinf(got[1]).all() and np.isnan(got[4]).all() and np.isneginf(got[7]).all()
    assert (np.delete(got, [1, 4, 7], axis=0) == K).all()
    relu = B.Linear(n, K, N, dt, "relu")
    relu.forward(x, w, y)
    got = y.float().cpu().numpy()
    assert np.isposinf(got[1]).all() and np.isnan(got[4]).all() and (got[7] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K", [(40, 24), (40, 600)])
def test_dy_that_is_not_finite_leaves_nothing_where_relu_is_closed(torch, B, dtype, n, K):
    dt, N = dtype_of(torch, dtype), 32
    x, w = torch.ones((n, K), dtype=dt, device="cuda"), torch.ones((N, K), dtype=dt, device="cuda")
    w[::2] = -1                                                  # z < 0 in the even columns
    dy = torch.ones((n, N), dtype=dt, device="cuda")
    dy[1, 2], dy[3, 4], dy[5, 6] = float("inf"), float("nan"), float("-inf")
    lay = B.Linear(n, K, N, dt, "relu", "before")
    y, saved, dz = (torch.empty((n, N), dtype=dt, device="cuda") for _ in range(3))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, dtype=dt, device="cuda")
    lay.forward(x, w, y, residual=torch.zeros_like(y), saved=saved)
    lay.backward(dy, x, w, saved, dx, dw, db, dz)
    want = (torch.arange(N, device="cuda") % 2).to(dt)
    assert torch.equal(dz, want.expand(n, N)) and torch.equal(db, n * want)
    assert torch.equal(dx, torch.full_like(dx, N / 2)) and torch.equal(dw, (n * want)[:, None].expand(N, K))


def test_gradients_match_differences(torch, B):
    """(L(p + h d) - L(p - h d)) / 2h of L = sum(dy y), in 64 bits, against the gradient's product with d."""
    n, K, N, G = 60, 20, 28, 3
    for act, mode in (("gelu", "before"), ("silu", "after"), ("none", "none")):
        rng = np.random.default_rng(11)
        f = lambda *s: rng.standard_normal(s).astype(np.float32)      # noqa: E731
        x, w, b, r, dy = f(n, K), f(G, N, K), f(G, N), f(n, N), f(n, N)
        group = rng.integers(0, G, n).astype(np.int32)
        dev = [torch.from_numpy(t).cuda() for t in (x, w, b, r, dy)]
        rg = B.RowGroups(n, G)
        rg.build(torch.from_numpy(group).cuda())
        lay = B.Linear(n, K, N, torch.float32, act, mode, G)
        y, saved, dx = torch.empty(n, N, device="cuda"), torch.empty(n, N, device="cuda"), torch.empty(n, K, device="cuda")
        dw, db = torch.empty(G, N, K, device="cuda"), torch.empty(G, N, device="cuda")
        dr = torch.empty(n, N, device="cuda") if mode == "before" else None
        lay.forward(dev[0], dev[1], y, dev[2], dev[3] if mode != "none" else None, saved, rg)
        lay.backward(dev[4], dev[0], dev[1], saved, dx, dw, db, dr, rg)
        grads = [t.double().cpu().numpy() for t in (dx, dw, db)] + [dr.double().cpu().numpy() if dr is not None else None]
        p = [t.astype(np.float64) for t in (x, w, b, r)]

        def loss(q):
            z = np.einsum("nk,nok->no", q[0], q[1][group]) + q[2][group] + (q[3] if mode == "before" else 0)
            return (dy * (act64(act, z)[0] + (q[3] if mode == "after" else 0))).sum()
        for i, grad in enumerate(grads):
            if grad is None:
                continue
            d, h = rng.standard_normal(p[i].shape), 1e-5
            up, down = list(p), list(p)
            up[i], down[i] = p[i] + h * d, p[i] - h * d
            slope = (loss(up) - loss(down)) / (2 * h)
            # the gradient's own error: some 30 roundings of fp32 on each of its terms; the difference's: h^2 of the third derivative
            assert abs(slope - (grad * d).sum()) <= 1e-4 * np.abs(grad * d).sum() / np.sqrt(d.size) + 1e-5 * np.abs(grad * d).sum()


def test_repeated_calls_give_the_same_bits_and_leave_inputs_alone(torch, B):
    n, K, N, G = 20_000, 72, 130, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, dy = (torch.randn(s, device="cuda", generator=g) for s in ((n, K), (G, N, K), (n, N)))
    of = torch.randint(0, G, (n,), device="cuda", generator=g, dtype=torch.int32)
    rg = B.RowGroups(n, G)
    lay = B.Linear(n, K, N, torch.float32, "silu", "none", G)
    keep = [t.clone() for t in (x, w, dy)]
    outs = []
    for _ in range(3):
        y, saved, dx, dw, db = (torch.empty(s, device="cuda") for s in ((n, N), (n, N), (n, K), (G, N, K), (G, N)))
        rg.build(of)
        lay.forward(x, w, y, saved=saved, groups=rg)
        lay.backward(dy, x, w, saved, dx, dw, db, groups=rg)
        outs.append([t.clone() for t in (y, dx, dw, db, rg.rows)])
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], o))
    assert all(torch.equal(a, b) for a, b in zip(keep, (x, w, dy)))


def test_residual_may_be_the_output_and_dz_may_be_dy(torch, B):
    n, K, N = 100, 30, 50
    x, w, r, dy = (torch.randn(s, device="cuda") for s in ((n, K), (N, K), (n, N), (n, N)))
    lay = B.Linear(n, K, N, torch.float32, "silu", "before")
    y, saved, dx, dw, dr = (torch.empty(s, device="cuda") for s in ((n, N), (n, N), (n, K), (N, K), (n, N)))
    lay.forward(x, w, y, residual=r, saved=saved)
    lay.backward(dy, x, w, saved, dx, dw, dresidual=dr)
    y2, d2, dx2, dw2 = r.clone(), dy.clone(), torch.empty_like(dx), torch.empty_like(dw)
    lay.forward(x, w, y2, residual=y2)
    lay.backward(d2, x, w, saved, dx2, dw2, dresidual=d2)
    for a, b in ((y, y2), (dr, d2), (dx, dx2), (dw, dw2)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,act,mode", [("f32", "silu", "none"), ("bf16", "relu", "before")])
@pytest.mark.parametrize("n,K,N,groups", [(25_000, 250, 40, 0), (25_500, 200, 33, 3), (900, 500, 70, 2), (300, 512, 130, 0)])
def test_several_tiles_of_dx_columns(torch, B, dtype, act, mode, n, K, N, groups):
    run_layer(torch, B, dtype, n, K, N, act, mode, groups=groups, seed=21)


@pytest.mark.parametrize("dtype,act", [("f32", "silu"), ("f32", "relu"), ("bf16", "relu"), ("bf16", "gelu")])
@pytest.mark.parametrize("n,K,N,groups", [(700, 100, 300, 0), (5485, 128, 520, 0), (900, 65, 260, 4), (33_000, 128, 70, 0)])
def test_dz_in_the_place_of_dy_where_dx_has_more_than_one_tile_of_columns(torch, B, dtype, act, n, K, N, groups):
    dt, G = dtype_of(torch, dtype), max(groups, 1)
    x, w, dy = (torch.randn(s, device="cuda").to(dt) for s in ((n, K), (G, N, K), (n, N)))
    w = w if groups else w[0]
    rg = None
    if groups:
        rg = B.RowGroups(n, groups)
        rg.build(torch.randint(-1, groups, (n,), dtype=torch.int32, device="cuda"))
    lay = B.Linear(n, K, N, dt, act, "before", groups)
    y, saved, dr = (torch.empty((n, N), dtype=dt, device="cuda") for _ in range(3))
    lay.forward(x, w, y, residual=dy, saved=saved, groups=rg)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    lay.backward(dy, x, w, saved, dx, dw, dresidual=dr, groups=rg)
    d2, dx2, dw2 = dy.clone(), torch.empty_like(dx), torch.empty_like(dw)
    lay.backward(d2, x, w, saved, dx2, dw2, dresidual=d2, groups=rg)
    for a, b in ((dr, d2), (dx, dx2), (dw, dw2)):
        assert torch.equal(a, b)


def test_another_stream_than_the_current_one(torch, B):
    s = torch.cuda.Stream()
    run_layer(torch, B, "bf16", 3000, 100, 72, "gelu", "before", seed=12, stream=s)
    run_layer(torch, B, "f32", 500, 100, 72, "gelu", "before", groups=3, seed=13, stream=s)


def test_groups_built_on_another_stream_before_the_current_one_has_cleared_them(torch, B):
    n, group = 3000, torch.randint(0, 5, (3000,), dtype=torch.int32, device="cuda")
    want = torch.cat([torch.zeros(1, dtype=torch.int64), torch.bincount(group.cpu(), minlength=5).cumsum(0)])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)               # some ms of the current stream, in front of the zeros
    rg = B.RowGroups(n, 5)
    rg.build(group, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(rg.offsets.cpu().long(), want)


def test_rows_beyond_four_gigabytes(torch, B):
    """Row strides that take the last rows' addresses past 32 bits, of bytes and (bf16) of values."""
    n, K, N, stride = 70_000, 16, 24, 64_000
    big = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")        # 9 GB
    x = big.view(n, stride)[:, :K]
    y = big.view(n, stride)[:, 1024: 1024 + N]
    x.copy_(torch.randn(n, K, device="cuda"))
    w = torch.randn(N, K, device="cuda").to(torch.bfloat16)
    dy = big.view(n, stride)[:, 2048: 2048 + N]
    dy.copy_(torch.randn(n, N, device="cuda"))
    dx = big.view(n, stride)[:, 4096: 4096 + K]
    lay = B.Linear(n, K, N, torch.bfloat16)
    dw = torch.empty_like(w)
    lay.forward(x, w, y)
    lay.backward(dy, x, w, dx=dx, dweight=dw)
    x64, w64, dy64 = x.double(), w.double(), dy.double()
    for got, want, mass in ((y, x64 @ w64.t().contiguous(), x64.abs() @ w64.abs().t().contiguous()),
                            (dx, dy64 @ w64, dy64.abs() @ w64.abs()),
                            (dw, dy64.t().contiguous() @ x64, dy64.abs().t().contiguous() @ x64.abs())):
        k = K if got is y else N if got is dx else n
        bound = (k + 4) * U * mass + 2.0 ** -8 * 1.01 * want.abs() + 1e-30
        assert bool(((got.double() - want).abs() <= bound).all())


def test_captured_calls_replay(torch, B):
    n, K, N, G = 3000, 40, 72, 4
    x, w, dy = (torch.randn(s, device="cuda") for s in ((n, K), (G, N, K), (n, N)))
    of = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    rg, lay = B.RowGroups(n, G), B.Linear(n, K, N, torch.float32, "gelu", "none", G)
    y, saved, dx, dw, db = (torch.empty(s, device="cuda") for s in ((n, N), (n, N), (n, K), (G, N, K), (G, N)))

    def step():
        rg.build(of)
        lay.forward(x, w, y, saved=saved, groups=rg)
        lay.backward(dy, x, w, saved, dx, dw, db, groups=rg)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.normal_()
        of.copy_(torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db, rg.rows, rg.offsets)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw, db, rg.rows, rg.offsets))), i


def test_the_binding_refuses_what_does_not_fit(torch, B):
    lay, typed = B.Linear(10, 8, 4), B.Linear(10, 8, 4, num_groups=2)
    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)      # noqa: E731
    x, w, y = f(10, 8), f(4, 8), f(10, 4)
    rg = B.RowGroups(10, 2)
    rg.build(f(9, dtype=torch.int32))
    for bad in (lambda: lay.forward(f(11, 8), w, f(11, 4)), lambda: lay.forward(f(10, 7), w, y), lambda: lay.forward(x, f(8, 4), y),
                lambda: lay.forward(x.bfloat16(), w, y), lambda: lay.forward(x.cpu(), w, y), lambda: lay.forward(f(8, 10).t(), w, y),
                lambda: lay.forward(x, w, y, groups=rg), lambda: typed.forward(x, f(2, 4, 8), y), lambda: lay.forward(x, w, f(9, 4)),
                lambda: typed.forward(x, f(2, 4, 8), y, groups=rg), lambda: lay.forward(x, w, y, bias=f(5)),
                lambda: lay.backward(f(1, 1).expand(10, 4), x, w, dx=f(10, 8)), lambda: B.Linear(10, 8, 4, torch.float16),
                lambda: B.Linear(10, 8, 4, activation="tanh"), lambda: rg.build(f(11, dtype=torch.int32)),
                lambda: rg.build(f(10, dtype=torch.int64)), lambda: rg.build(f(10, dtype=torch.int32), n=11)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.Linear(10, 0, 4), lambda: B.Linear(10, 8, 4, num_groups=5000), lambda: B.RowGroups(10, 0),
                lambda: lay.forward(x, w, y, residual=f(10, 4)), lambda: lay.backward(y, x, w, dx=x, dresidual=y)):
        with pytest.raises(B.BglError):
            bad()


@pytest.mark.parametrize("most,n,groups", [(524_800, 524_288, 8), (560_000, 524_288, 1024), (655_361, 655_360, 100)])
def test_room_for_many_rows_is_room_for_fewer(torch, B, most, n, groups):
    """A batch a little smaller than the largest is cut into more tiles than that one."""
    rg = B.RowGroups(most, groups)
    of = torch.randint(-1, groups, (n,), dtype=torch.int32, device="cuda")
    rg.build(of)
    key = of.cpu().numpy()
    key = np.where(key < 0, groups, key)
    assert np.array_equal(rg.rows.cpu().numpy(), np.argsort(key, kind="stable"))
    assert np.array_equal(rg.offsets.cpu().numpy(), np.searchsorted(np.sort(key), np.arange(groups + 1)))


def single_values(torch, B, dtype, act, z):
    """act(z) and its slope as a layer of one weight of 1 makes them: the product is exact, so nothing else has a part in it."""
    dt = dtype_of(torch, dtype)
    x = torch.from_numpy(z.astype(np.float32)).to(dt).cuda()[:, None]
    lay, one = B.Linear(len(z), 1, 1, dt, act), torch.ones((1, 1), dtype=dt, device="cuda")
    y, saved, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    lay.forward(x, one, y, saved=saved)
    lay.backward(torch.ones_like(x), x, one, saved, dx)
    return tuple(t.double().cpu().numpy()[:, 0] for t in (x, y, dx))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_are_right_to_the_last_places_in_the_tails_too(torch, B, dtype, act):
    """Relative to the value, not to 1.  fp32, in unit roundoffs u: gelu's Phi(-|z|) is the product of an exponential (its hardware 2^x 2, the
    rest of its argument and the product 3), a numerator and a denominator (2 each), a reciprocal (2) and two products: 16 with the
    rational function's own 0.1 and z; silu 10 for exponential 5, sum, reciprocal 2 and product.  Slopes: the same of each term; silu's 1 - p has p's error.  bf16:
    2^-15 of the value, and the type's rounding; the slope there sees z rounded to a half."""
    from scipy.special import erfc
    rng = np.random.default_rng(31)
    far = 12.5 if act == "gelu" else 80.0
    z = np.concatenate([rng.uniform(-far, far, 60_000), rng.uniform(-1, 1, 30_000), 2.0 ** rng.uniform(-30, 3, 5000), -2.0 ** rng.uniform(-30, 3, 5000)])
    z, y, dx = single_values(torch, B, dtype, act, z)
    if act == "gelu":
        p, places = 0.5 * erfc(-z / np.sqrt(2)), 16
        bell = z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        slope, mass = p + bell, p + np.abs(bell)
    else:
        p, places = 1 / (1 + np.exp(-z)), 10
        slope, mass = p * (1 + z * (1 - p)), p * (1 + np.abs(z) * (1 - p)) + np.abs(z) * p * p
    want = z * p
    relative = (places + 1) * U if dtype == "f32" else 2.0 ** -8 * 1.001 + 2.0 ** -15
    off = np.abs(y - want) / (np.abs(want) * relative + 2.0 ** -120)
    assert off.max() <= 1, f"value: {off.max():.1f} times the bound at z = {z[off.argmax()]}"
    e = (places + 2) * U * mass if dtype == "f32" else 2.0 ** -8 * 1.001 * np.abs(slope) + 2.0 ** -15 * mass + 0.8 * (2.0 ** -11 * np.abs(z) + 2.0 ** -24)
    off = np.abs(dx - slope) / (e + 2.0 ** -120)
    assert off.max() <= 1, f"slope: {off.max():.1f} times the bound at z = {z[off.argmax()]}"


def test_tensors_that_require_gradients_are_refused_rather_than_their_gradients_lost(torch, B):
    n, K, N = 70, 20, 12
    lay = B.Linear(n, K, N, torch.float32, "silu", "before")
    x, w, b, r, dy = (torch.randn(s, device="cuda") for s in ((n, K), (N, K), (N,), (n, N), (n, N)))
    y, saved, dx, dr, dw, db = (torch.empty_like(t) for t in (dy, dy, x, dy, w, b))
    given = dict(x=x, weight=w, bias=b, residual=r)
    for name in given:
        some = {k: t.clone().requires_grad_() if k == name else t for k, t in given.items()}
        with pytest.raises(ValueError, match="gradients"):
            lay.forward(y=y, **some)
        with torch.no_grad():
            lay.forward(y=y, **some)

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b, r):
            out = torch.empty_like(r)
            lay.forward(x, w, out, b, r, saved)
            ctx.save_for_backward(x, w)
            return out

        @staticmethod
        def backward(ctx, d):
            lay.backward(d.contiguous(), *ctx.saved_tensors, saved, dx, dw, db, dr)
            return dx.clone(), dw.clone(), db.clone(), dr.clone()
    leaves = [t.clone().requires_grad_() for t in (x, w, b, r)]
    Layer.apply(*leaves).backward(dy)
    lay.forward(x, w, y, b, r, saved)
    lay.backward(dy, x, w, saved, dx, dw, db, dr)
    for leaf, want in zip(leaves, (dx, dw, db, dr)):
        assert torch.equal(leaf.grad, want)


def rows_for_large_tiles(columns):
    """The fewest rows whose product of `columns` columns the library makes in tiles of 128 rows, by the rule that its source states today."""
    import os
    import re
    from paper_2112_08541_amd import buildlib
    text = open(os.path.join(buildlib.CSRC, "bgl_linear.hip")).read()
    least, = re.search(r"bool large_tiles\(int64_t n, int64_t cols\) \{ return ceil_div\(n, 128\) \* ceil_div\(cols, 128\) >= (\d+); \}", text).groups()
    return (-(-int(least) // -(-columns // 128)) - 1) * 128 + 1


def exact_layer(torch, B, dtype, n, K, N, act, mode, groups=0, in_place=False, want_dx=True, seed=0):
    """A layer over small whole numbers: all sums are whole and below 2^24, so every output has one right value, which is then
    rounded to the type once; a row or a column left out, or counted twice, is another one."""
    dt, G = dtype_of(torch, dtype), max(groups, 1)
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + n)
    whole = lambda *s: torch.randint(-2, 3, s, generator=gen, device="cuda").to(dt)      # noqa: E731
    x, w, b, dy = whole(n, K), whole(G, N, K), whole(G, N), whole(n, N)
    r = whole(n, N) if mode != "none" else None
    group, rg = torch.zeros(n, dtype=torch.int64, device="cuda"), None
    if groups:
        of = torch.randint(-1, groups, (n,), generator=gen, dtype=torch.int32, device="cuda")
        rg = B.RowGroups(n, groups)
        rg.build(of)
        group = of.long()
    z = torch.zeros((n, N), dtype=torch.float64, device="cuda")
    members = [torch.nonzero(group == g).squeeze(1) for g in range(G)]
    for g, at in enumerate(members):
        z[at] = x[at].double() @ w[g].double().t().contiguous() + b[g].double()
    if mode == "before":
        z += r.double()
    y64 = z.clamp(min=0) if act == "relu" else z
    if mode == "after":
        y64 = y64 + r.double()
    dz = dy.double() * (z > 0) if act == "relu" else dy.double()
    dx64 = torch.zeros((n, K), dtype=torch.float64, device="cuda")
    dw64, db64 = torch.zeros((G, N, K), dtype=torch.float64, device="cuda"), torch.zeros((G, N), dtype=torch.float64, device="cuda")
    for g, at in enumerate(members):
        dx64[at] = dz[at] @ w[g].double()
        dw64[g] = dz[at].t().contiguous() @ x[at].double()
        db64[g] = dz[at].sum(0)
    assert max(float(t.abs().max()) for t in (z, dx64, dw64, db64)) < 2 ** 24
    lay = B.Linear(n, K, N, dt, act, mode, groups)
    lay.workspace = B._workspace(lay._bytes(n)).fill_(0xFF)      # NaN wherever nothing is written
    y, dw, db = torch.full_like(dy, float("nan")), torch.full_like(w, float("nan")), torch.full_like(b, float("nan"))
    saved = torch.full_like(dy, float("nan")) if act != "none" else None
    dx = torch.full_like(x, float("nan")) if want_dx else None
    dres = None if mode != "before" else dy if in_place else torch.full_like(dy, float("nan"))
    one = lambda t: t if groups else t[0]      # noqa: E731
    lay.forward(x, one(w), y, one(b), r, saved, rg)
    lay.backward(dy, x, one(w), saved, dx, one(dw), one(db), dres, rg)
    for name, got, want in (("y", y, y64), ("dx", dx, dx64), ("dresidual", dres, dz), ("dweight", dw, dw64), ("dbias", db, db64)):
        if got is not None:
            wrong = got != want.to(dt)
            assert not bool(wrong.any()), f"{name}: {int(wrong.sum())} of {wrong.numel()} values, the first at {torch.nonzero(wrong)[0].tolist()}"


# one width for each number of blocks of 16 columns up to a tile's eight, whole and cut, and two tiles of columns
WIDTHS = [3, 16, 31, 45, 64, 77, 96, 100, 127, 250]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [0, 5])
@pytest.mark.parametrize("i", range(len(WIDTHS)))
def test_large_tiles_of_every_width(torch, B, dtype, i, groups):
    """Forward tiles as wide as N, those of dx as wide as K; dz made within dx (relu) and none (no activation)."""
    K, N = WIDTHS[i], WIDTHS[-1 - i]
    n = rows_for_large_tiles(min(K, N)) + 45
    exact_layer(torch, B, dtype, n, K, N, "relu", "before", groups, seed=1)
    exact_layer(torch, B, dtype, n, K, N, "none", "after", groups, seed=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [0, 5])
@pytest.mark.parametrize("K,N", [(100, 256), (512, 256), (300, 40), (260, 130), (128, 70), (200, 33)])
def test_large_tiles_with_dz_within_dx_apart_and_in_the_place_of_dy(torch, B, dtype, K, N, groups):
    """dx of one tile of columns, of two, and of so many that dz is made before it; the same with dz in dy's place."""
    n = max(rows_for_large_tiles(K), rows_for_large_tiles(N)) + 83
    exact_layer(torch, B, dtype, n, K, N, "relu", "before", groups, seed=3)
    exact_layer(torch, B, dtype, n, K, N, "relu", "before", groups, in_place=True, seed=4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [0, 40])
@pytest.mark.parametrize("width", WIDTHS)
def test_no_row_is_left_out_of_a_weight_gradient_of_any_width(torch, B, dtype, width, groups):
    """The narrower side of dW's tiles as wide as `width`, on either side of the product; small tiles of the other products too."""
    n = rows_for_large_tiles(128) // 3
    exact_layer(torch, B, dtype, n, width, 300, "none", "none", groups, want_dx=False, seed=5)
    exact_layer(torch, B, dtype, n, 140, width, "relu", "before", groups, seed=6)
    exact_layer(torch, B, dtype, n, width, 60, "none", "none", groups, seed=7)


@pytest.mark.parametrize("dtype,act", [("f32", "gelu"), ("f32", "silu"), ("bf16", "gelu"), ("bf16", "silu")])
@pytest.mark.parametrize("K,N,groups", [(100, 96, 0), (300, 160, 0), (40, 256, 6)])
def test_gradients_of_smooth_activations_miss_no_row(torch, B, dtype, act, K, N, groups):
    """dresidual is dz as the products read it, so dx and dW are its products but for their own sums and the type's rounding.  bf16 layers add db up
    before dz is rounded: against the slopes of z as it was kept, a half, within 2^-15 of each term (the activation's) and the sum's error.  The sums' errors
    are taken as 8 sqrt(rows) u of the largest partial sum a random walk of the terms reaches, not as the linear worst case, which hides hundreds of rows."""
    dt, G = dtype_of(torch, dtype), max(groups, 1)
    n = max(rows_for_large_tiles(K), rows_for_large_tiles(N)) + 17
    gen = torch.Generator(device="cuda").manual_seed(n)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")      # noqa: E731
    x, w, b, r, dy = f(n, K).to(dt), (f(G, N, K) / K ** 0.5).to(dt), f(G, N).to(dt), f(n, N).to(dt), f(n, N).to(dt)
    group, rg = torch.zeros(n, dtype=torch.int64, device="cuda"), None
    if groups:
        of = torch.randint(-1, groups, (n,), generator=gen, dtype=torch.int32, device="cuda")
        rg, group = B.RowGroups(n, groups), of.long()
        rg.build(of)
    lay = B.Linear(n, K, N, dt, act, "before", groups)
    y, saved, dres, dx, dw, db = (torch.full_like(t, float("nan")) for t in (dy, dy, dy, x, w, b))
    one = lambda t: t if groups else t[0]      # noqa: E731
    lay.forward(x, one(w), y, one(b), r, saved, rg)
    lay.backward(dy, x, one(w), saved, dx, one(dw), one(db), dres, rg)
    v = U if dtype == "f32" else 2.0 ** -8
    z = (saved.view(torch.float16) if dtype == "bf16" else saved).double()
    if act == "gelu":
        p = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
        bell = z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
        slope, mass = p + bell, p + bell.abs()
    else:
        p = torch.sigmoid(z)
        slope, mass = p * (1 + z * (1 - p)), p * (1 + z.abs() * (1 - p)) + z.abs() * p * p
    dz, d64 = dy.double() * slope, dres.double()
    places = 20 * U if dtype == "f32" else 2.0 ** -15
    near = lambda name, got, want, bound: _near(torch, name, got, want, bound)      # noqa: E731
    near("dresidual", dres, dz, v * 1.001 * dz.abs() + places * dy.double().abs() * mass + 1e-30)
    for g in range(G):
        at = torch.nonzero(group == g).squeeze(1)
        x64, w64, d = x[at].double(), w[g].double(), d64[at]
        z64 = x64 @ w64.t().contiguous() + b[g].double() + r[at].double()
        kept = 2.0 ** -11 if dtype == "bf16" else U
        near("z", (saved.view(torch.float16) if dtype == "bf16" else saved)[at], z64,
             kept * 1.001 * z64.abs() + (K + 4) * U * (x64.abs() @ w64.abs().t().contiguous() + b[g].double().abs() + r[at].double().abs()) + 2.0 ** -24)
        near("dx", dx[at], d @ w64, v * 1.001 * (d @ w64).abs() + (N + 4) * U * (d.abs() @ w64.abs()) + 1e-30)
        walk = (d.square().t().contiguous() @ x64.square()).sqrt()
        near("dweight", dw[g], d.t().contiguous() @ x64, v * 1.001 * (d.t().contiguous() @ x64).abs() + 8 * len(at) ** 0.5 * U * walk + 1e-30)
        want = dz[at].sum(0)
        near("dbias", db[g], want, v * 1.001 * want.abs() + 8 * len(at) ** 0.5 * U * dz[at].square().sum(0).sqrt()
             + places * (dy[at].double().abs() * mass[at]).sum(0) + 1e-30)


def _near(torch, name, got, want, bound):
    off = ((got.double() - want).abs() / bound)
    assert bool(torch.isfinite(got).all()) and float(off.max()) <= 1.0, f"{name}: {float(off.max()):.2f} times the bound"


def test_a_layer_without_its_weight_is_the_librarys_error(torch, B):
    x, y = torch.zeros((3, 8), device="cuda"), torch.zeros((3, 4), device="cuda")
    with pytest.raises(B.BglError, match="weight"):
        B.Linear(3, 8, 4).forward(x, None, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_of_values_that_are_not_finite(torch, B, dtype, act):
    """z times a probability: infinity stays, minus infinity meets 0 and is not a number, as in the formula; nothing else is touched."""
    z = np.array([np.inf, np.nan, -np.inf, 1e30, -1e30, 0.0, -0.0])
    _, y, _ = single_values(torch, B, dtype, act, z)
    assert np.isposinf(y[0]) and np.isnan(y[1]) and np.isnan(y[2]) and abs(y[3] / 1e30 - 1) < 0.01 and (y[4:] == 0).all()
