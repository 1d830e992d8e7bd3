"""Losses over class scores at sizes that are laid out for large tiles, of operands whose values are of very different sizes, with the bounds of test_gpu_classes_large.py:
no row or class may lose what it has because another one is large."""
import pytest

from test_gpu_classes import B, inputs, torch  # noqa: F401
from test_gpu_classes_large import check_large

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("up", [12, 20, 31, 60])
def test_columns_of_different_sizes(torch, B, up):
    """A column of x far above the others (seconds since 1970 beside shares of 1) with weights as far below: every product counts."""
    n, D, C = 600, 352, 9_600
    x, w, b, labels, teacher = inputs(torch, "f32", n, D, C, 2, seed=24)
    x[:, 3] *= 2.0 ** up
    w[:, 3] *= 2.0 ** -up
    check_large(torch, B, "f32", (x, w, b, labels, teacher), t=1.5, s=1.0 / n, st=0.5 / n)
