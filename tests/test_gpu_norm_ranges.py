"""Layer norm of rows whose values hardly differ, or not at all, beside their size, up to the largest numbers, against the definition in 64 bits.

The bounds are those of test_gpu_norm.py without its u |mean| r: the mean counts in the values' differences from it alone.  Where these are no more than the last places
of the values, the mean of x - m has up to 2 sigma of absolute values (m is the nearest number to the mean, and differences are whole last places), so it is off by 60 u
sigma, squares less the mean's square by 70 u of the variance, r by 40 u; a mean within 16 sigma of 0 is kept in 32 bits for the backward call, 16 u.  Together H = 40 u |h| + 80 u.
Rows of equal values have h = 0, whatever they are: y is the bias."""
import numpy as np
import pytest

from test_gpu_norm import B, U, V, Reference, check, dtype_of, np64, run_both, torch  # noqa: F401

pytestmark = pytest.mark.gpu


class Near(Reference):
    def __init__(self, x, w, b, eps, v):
        n, width = x.shape
        self.x, self.v, self.width = x, v, width
        self.g = np.ones(width) if w is None else w
        bias = np.zeros(width) if b is None else b
        d = x - x[:, :1]
        d = d - d.mean(1, keepdims=True)
        d = np.where((x == x[:, :1]).all(1, keepdims=True), 0.0, d)
        self.r = 1 / np.sqrt((d ** 2).mean(1, keepdims=True) + eps)
        self.h = d * self.r
        self.H = 40 * U * np.abs(self.h) + 80 * U
        self.y = self.h * self.g + bias
        self.y_bound = np.abs(self.g) * self.H + 2 * U * (np.abs(self.h * self.g) + np.abs(bias)) + 1.01 * v * np.abs(self.y) + 1e-37


def others(torch, kind, n, width, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    return rnd, [v.to(dtype_of(torch, kind)) for v in (1 + 0.3 * rnd(width), 0.5 * rnd(width), rnd(n, width))]


def check_rows(torch, B, kind, x, w, b, dy, eps):
    ref = Near(np64(x), np64(w), np64(b), eps, V[kind])
    got = run_both(torch, B, kind, x, w, b, dy, eps)
    check("y", got["y"], ref.y, ref.y_bound)
    for name, (value, bound) in zip(("dx", "dweight", "dbias"), ref.gradients(np64(dy))):
        check(name, got[name], value, bound + 2.0 ** -140)      # (gradients of huge rows are near the smallest numbers)
    return got


WIDTHS = [1, 2, 5, 100, 256, 700, 1_024, 1_500, 2_048, 5_000, 9_001, 16_384]
VALUES = [0.0, 1e-30, -3.3, 1e4, 1e8, -1e12, 1e19, -1e30, 2e34, 1e36, -1e37, 1e38, 3.38e38]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("eps", [1e-5, 1e-12, 100.0])
def test_rows_of_equal_values(torch, B, kind, width, eps):
    n = 2 * len(VALUES)
    rnd, (w, b, dy) = others(torch, kind, n, width, seed=width)
    x = rnd(n, width)
    x[::2] = torch.tensor(VALUES, device="cuda")[:, None]      # (beside ordinary rows)
    x = x.to(dtype_of(torch, kind))
    assert x.isfinite().all()
    got = check_rows(torch, B, kind, x, w, b, dy, eps)
    assert torch.equal(got["y"][::2], b.expand(len(VALUES), width))


@pytest.mark.parametrize("width", WIDTHS[1:])
@pytest.mark.parametrize("at", [1.0, 1e5, 1e30, 3e37])
def test_rows_that_differ_in_their_last_places(torch, B, width, at):
    """A value one place off, two kinds of values, a few places in any order."""
    n = 9
    rnd, (w, b, dy) = others(torch, "f32", n, width, seed=width + 1)
    place = torch.full((), at, device="cuda")
    step = torch.nextafter(place, place * 2) - place
    off = torch.zeros((n, width), device="cuda")
    off[0, 0], off[1, -1], off[2, width // 2], off[3, :width // 2] = 1, 1, -3, 1
    off[4:] = (rnd(n - 4, width) * torch.tensor([0.5, 1.0, 3.0, 50.0, 1_000.0], device="cuda")[:, None]).round()
    check_rows(torch, B, "f32", at + off * step, w, b, dy, 1e-5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", [2, 100, 700, 1_500, 5_000])
@pytest.mark.parametrize("shift", [10.0, 30.0, 1e3, 1e4, 1e5, 1e6])
def test_rows_far_from_zero(torch, B, kind, width, shift):
    """Forward and backward are as near as those of rows around 0, and the rows beside them."""
    n = 23
    rnd, (w, b, dy) = others(torch, kind, n, width, seed=width + 2)
    x = rnd(n, width)
    x[::2] += shift * (1 + rnd(12, 1).abs())
    check_rows(torch, B, kind, x.to(dtype_of(torch, kind)), w, b, dy, 1e-5)


def test_places_behind_the_row(torch, B):
    """Widths that leave room in the last thread's pieces, of rows whose mean over their deviation is beyond the type."""
    for width in (1, 3, 9, 65, 513, 1_025, 4_100):
        rnd, (w, b, dy) = others(torch, "f32", 4, width, seed=width)
        x = torch.tensor([3e38, -2e37, 4e33, 1.0], device="cuda")[:, None].expand(4, width).contiguous()
        check_rows(torch, B, "f32", x, w, b, dy, 1e-12)


def test_a_stream_of_another_device_is_refused(torch, B):
    """As far as one device can show it; nothing is launched."""
    class Other:
        device_index, cuda_stream = torch.cuda.current_device() + 1, 0
    x, w, labels = torch.zeros((4, 8), device="cuda"), torch.zeros((5, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    pairs, norm, loss = torch.zeros((4, 2), device="cuda"), B.LayerNorm(4, 8), B.ClassLoss(4, 8, 5)
    for call in (lambda: norm.forward(x, x, stream=Other), lambda: norm.backward(x, x, pairs, dx=x, stream=Other),
                 lambda: loss.forward(x, w, labels=labels, stream=Other), lambda: loss.backward(x, w, pairs, labels=labels, dx=x, stream=Other)):
        with pytest.raises(ValueError, match="stream of device"):
            call()
    side = torch.cuda.Stream()
    norm.forward(x, x, stream=side)
    torch.cuda.synchronize()
