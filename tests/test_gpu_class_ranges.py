"""Losses over class scores at sizes that are laid out for large tiles, of operands whose values are of very different sizes, with the bounds of test_gpu_classes_large.py:
no row or class may lose what it has because another one is large."""
import pytest

from test_gpu_classes import B, inputs, torch  # noqa: F401
import test_gpu_classes_large as large
from test_gpu_classes_large import check_large

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("up", [10, 14, 20, 36, 90])
def test_a_row_far_above_the_others(torch, B, kind, up):
    n, D, C = 600, 352, 9_600
    x, w, b, labels, teacher = inputs(torch, kind, n, D, C, 2, seed=21)
    x[5] *= 2.0 ** up
    labels[5] = 77
    for some in (None, teacher):
        check_large(torch, B, kind, (x, w, b, labels, some), t=2.0, s=1.0 / n, st=0.5 / n if some else 0.0, far=up < 12)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("up", [14, 40, 90])
def test_a_class_far_above_the_others(torch, B, kind, up):
    """Where x is 0, so that the scores are as before."""
    n, D, C = 600, 352, 9_600
    x, w, b, labels, _ = inputs(torch, kind, n, D, C, 0, seed=22)
    x[:, :8] = 0
    w[7, :8] *= 2.0 ** up
    check_large(torch, B, kind, (x, w, b, labels, None), s=1.0 / n, st=0.0)


@pytest.mark.parametrize("down", [30, 60, 105])
def test_rows_of_the_smallest_numbers(torch, B, down):
    """All of x so small that scores are the bias: dweight is as near as of others."""
    n, D, C = 600, 352, 9_600
    x, w, b, labels, _ = inputs(torch, "bf16", n, D, C, 0, seed=23)
    check_large(torch, B, "bf16", ((x.float() * 2.0 ** -down).bfloat16(), w, b, labels, None), s=1.0, st=0.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("up", [12, 20, 31, 60])
def test_columns_of_different_sizes(torch, B, kind, up):
    """A column of x far above the others (seconds since 1970 beside shares of 1) with weights as far below: every product counts."""
    n, D, C = 600, 352, 9_600
    x, w, b, labels, teacher = inputs(torch, kind, n, D, C, 2, seed=24)
    x[:, 3] *= 2.0 ** up
    w[:, 3] *= 2.0 ** -up
    check_large(torch, B, kind, (x, w, b, labels, teacher), t=1.5, s=1.0 / n, st=0.5 / n)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_weight_beyond_32_bits(torch, B, kind):
    large.test_a_weight_beyond_32_bits(torch, B, kind, 130)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [(128, 512, 40_003, 3), (129, 512, 40_003, 3), (129, 513, 41_003, 0), (20_001, 801, 128, 2), (20_001, 801, 129, 2), (160, 64, 200_003, 0)])
def test_borders(torch, B, kind, n, D, C, k):
    """From the small tiles' last row and class to the large ones' first."""
    check_large(torch, B, kind, inputs(torch, kind, n, D, C, k, seed=n + C, pad=n % 3), t=1.5, s=1.0 / n, st=0.5 / n if k else 0.0)
