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
@pytest.mark.parametrize("n,D,C,k", [(600, 352, 9_600, 0), (600, 352, 9_600, 3), (20_000, 800, 130, 0), (97, 640, 33_000, 2), (5_000, 400, 1_001, 4)])
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
