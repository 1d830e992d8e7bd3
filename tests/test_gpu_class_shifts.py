"""A softmax does not change when all of a row's scores are moved: losses and gradients of scores that lie far below or above 0, with the bounds of test_gpu_classes.py and
test_gpu_classes_large.py, on every way a row's sum comes together: in a tile, from the tiles' halves, from few parts, many, and the parts of many rows."""
import pytest

from test_gpu_classes import B, check_all, inputs, run, torch  # noqa: F401
from test_gpu_classes_large import check_large

pytestmark = pytest.mark.gpu

SHIFTS = [-90.0, -100.0, -1_000.0, -30_000.0, 1_000.0]


def moved(data, shift):
    x, w, b, labels, teacher = data
    return x, w, (b.float() + shift).to(b.dtype), labels, teacher


@pytest.mark.parametrize("shift", SHIFTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [
    (40, 20, 3, 0), (40, 20, 17, 0), (40, 20, 40, 0), (40, 20, 50, 3), (70, 16, 90, 0), (70, 16, 65, 2),         # one tile, some of its wavefronts without a class
    (9_000, 12, 10, 0), (9_000, 12, 40, 2),                                                                  # one tile, many rows
    (100, 30, 300, 3), (1, 24, 300, 0), (3, 24, 9_000, 0), (3, 24, 9_000, 5), (90, 30, 5_000, 0), (90, 30, 5_000, 9)])      # few parts, many, those of many rows
def test_scores_far_from_zero(torch, B, kind, n, D, C, k, shift):
    data = moved(inputs(torch, kind, n, D, C, k, seed=n + C), shift)
    check_all(torch, B, kind, data, t=2.0, s=0.4 / n, st=0.6 / n)
    if k:
        check_all(torch, B, kind, (*data[:3], None, data[4]), t=1.0, s=0.0, st=1.0 / n)


@pytest.mark.parametrize("shift", SHIFTS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [(600, 352, 9_600, 0), (600, 352, 9_600, 3), (20_000, 800, 130, 0), (131, 640, 33_000, 2), (5_000, 400, 1_001, 4)])
def test_large_calls(torch, B, kind, n, D, C, k, shift):
    check_large(torch, B, kind, moved(inputs(torch, kind, n, D, C, k, seed=n), shift), t=2.0, s=1.0 / n, st=0.5 / n if k else 0.0, far=True)


@pytest.mark.parametrize("t", [0.05, 0.1])
@pytest.mark.parametrize("shift", [0.0, -10.0, -100.0])
@pytest.mark.parametrize("n,D,C,k", [(40, 20, 40, 3), (100, 30, 300, 3), (3, 24, 9_000, 5), (90, 30, 5_000, 9), (600, 352, 9_600, 3)])
def test_low_temperatures(torch, B, n, D, C, k, shift, t):
    data = moved(inputs(torch, "f32", n, D, C, k, seed=n + 1), shift)
    checked = check_large if n * D * C >= 2e9 else check_all
    checked(torch, B, "f32", data, t=t, s=0.4 / n, st=0.6 / n)
    checked(torch, B, "f32", (*data[:3], None, data[4]), t=t, s=0.0, st=1.0 / n)


@pytest.mark.parametrize("shift", [-100.0, -1_000.0])
@pytest.mark.parametrize("n,D,C", [(50, 20, 300), (50, 20, 50), (90, 30, 5_000), (600, 352, 9_600)])
def test_classes_taken_out(torch, B, n, D, C, shift):
    """Whole tiles of classes with a bias of -inf, before, between and behind the others; a row for which no class is left has NaN."""
    x, w, b, labels, _ = moved(inputs(torch, "f32", n, D, C, 0, seed=5), shift)
    out = torch.zeros(C, dtype=torch.bool, device="cuda")
    for first, last in ((0.0, 0.1), (0.3, 0.6), (0.8, 1.0)):
        out[int(first * C):int(last * C)] = True
    b[out] = -float("inf")
    left = torch.nonzero(~out)[:, 0].int()
    labels[labels >= 0] = left[labels[labels >= 0].long() % len(left)]
    checked = check_large if n * D * C >= 2e9 else check_all
    got = checked(torch, B, "f32", (x, w, b, labels, None), s=1.0 / n, st=0.0)
    assert (got["dweight"][out] == 0).all() and (got["dbias"][out] == 0).all()
    b[:] = -float("inf")
    assert run(torch, B, "f32", x, w, b, labels, None, s=1.0 / n)["loss"][labels >= 0].isnan().all()


@pytest.mark.parametrize("C,at", [(300, 299), (257, 256), (50, 40), (5_000, 4_999)])
def test_a_class_that_is_nan_is_not_lost(torch, B, C, at):
    """Where it is alone in its part of a row, that part has no largest value."""
    x, w, b, labels, _ = inputs(torch, "f32", 70, 20, C, 0, seed=7)
    w[at:] = float("nan")
    labels[:] = 0
    assert run(torch, B, "f32", x, w, b, labels, None, s=1.0)["loss"].isnan().all()


HIGH = [2.0 ** 23, -2.0 ** 24, 2.0 ** 27, -2.0 ** 30, 2.0 ** 31, -2.0 ** 33, 2.0 ** 40, -2.0 ** 100]


@pytest.mark.parametrize("t", [1.0, 1024.0, 2.0 ** -10])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(50, 3), (50, 40), (70, 300), (90, 1_300), (1_300, 1_300), (9_000, 12)])
def test_scores_beyond_the_steps_of_their_exponents(torch, B, kind, n, C, t):
    """Scores as large as 2^100, a few steps of 1 or of their last place apart, beside ordinary ones.  The weight is the identity, so that scores are x and dx is dz; every row's own
    step makes its distribution anything from even to a single class.  Powers are right to 6 u and 2 u of their argument (which e^-a a <= 0.4 keeps below 1 u in q), sums of
    them to u for each of C / 16 + 40 steps and 8 u for each of the parts' 8 scalings: q to 2 (6 + 64) + C / 8 + 80 = 220 + C / 8 u, and so is a loss beside 4 u of itself."""
    u, dtype = 2.0 ** -24, torch.float32 if kind == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(C + n)
    high = torch.tensor(HIGH + [0.0], dtype=torch.float64, device="cuda")[torch.arange(n, device="cuda") % 9]
    place = 2.0 ** ((high.abs() + 1).log2().floor() - (23 if kind == "f32" else 7))
    step = torch.where(torch.arange(n, device="cuda") % 2 == 0, place.clamp(min=t / 2), place.clamp(min=1.0))
    z = high[:, None] - torch.randint(0, 9, (n, C), generator=g, device="cuda") * step[:, None] * high.sign()[:, None].where(high[:, None] != 0, torch.ones_like(high)[:, None])
    x = z.to(dtype)
    z = x.double()
    w = torch.eye(C, dtype=dtype, device="cuda")
    labels = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    classes = torch.stack([torch.randperm(C, generator=g, device="cuda")[:3] for _ in range(n)]).int()
    scores = torch.randint(-8, 8, (n, 3), generator=g, device="cuda") * (t / 4)
    off = (220 + C / 8) * u
    p = torch.zeros((n, C), dtype=torch.float64, device="cuda").scatter_(1, classes.long(), (scores.double() / t).softmax(1))
    logq, logq_t = z.log_softmax(1), (z / t).log_softmax(1)
    loss = -logq[torch.arange(n, device="cuda"), labels.long()]
    teacher_loss = t * t * (torch.special.xlogy(p, p) - p * logq_t).sum(1)
    one = torch.nn.functional.one_hot(labels.long(), C)
    for use, teacher, s, st in ((labels, None, 1.0, 0.0), (labels, (classes, scores), 1.0, 0.5), (None, (classes, scores), 0.0, 0.5)):
        got = run(torch, B, kind, x, w, None, use, teacher, t, s, st)
        if use is not None:
            assert ((got["loss"].double() - loss).abs() <= off + 4 * u * loss).all()
        if teacher is not None:
            assert ((got["teacher_loss"].double() - teacher_loss).abs() <= t * t * off + 8 * u * teacher_loss).all()
        dz = (s * (logq.exp() - one) if s else 0) + (st * t * (logq_t.exp() - p) if st else 0)
        v, each = (2.0 ** -8 if kind == "bf16" else 2.0 ** -24), (s + 2 * st * t) * off
        assert ((got["dx"].double() - dz).abs() <= 2.1 * v * dz.abs() + each).all()
        assert got["dbias"].isfinite().all() and got["dweight"].isfinite().all()
        want, size = dz.t() @ z, dz.abs().t().contiguous() @ z.abs()
        assert ((got["dweight"].double() - want).abs() <= 2.1 * v * size + (n + 8) * u * size + each * z.abs().sum(0) + v * want.abs()).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("t", [0.05, 3.0, 7.0])
@pytest.mark.parametrize("n,D,C,k", [(70, 30, 300, 8), (70, 30, 300, 9), (1_100, 20, 90, 8), (1_100, 20, 90, 40), (600, 352, 9_600, 5)])
def test_a_teachers_scores_far_from_zero(torch, B, kind, n, D, C, k, t):
    """Scores that are exact when moved, so that nothing changes when they are."""
    x, w, b, labels, teacher = inputs(torch, kind, n, D, C, k, seed=n + k)
    scores = (teacher[1] * 128).round() / 128
    want = run(torch, B, kind, x, w, b, labels, (teacher[0], scores), t, 0.4, 0.6)
    for move in (-30_000.0, 1_000.0, 60_000.0):
        got = run(torch, B, kind, x, w, b, labels, (teacher[0], scores + move), t, 0.4, 0.6)
        assert all(torch.equal(got[i], want[i]) for i in got), move
