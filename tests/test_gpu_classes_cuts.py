"""Losses over class scores at the borders between the tiles and launches that small calls choose from, with the bounds of test_gpu_classes.py."""
import pytest

from test_gpu_classes import B, check_all, inputs, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,D,C,k", [
    (8_192, 10, 16, 0), (8_192, 11, 17, 3), (9_000, 20, 32, 2), (8_200, 33, 33, 0), (8_200, 33, 64, 4), (8_191, 12, 64, 0), (8_193, 8, 65, 0),     # few classes of many rows
    (16, 40, 9_000, 3), (17, 40, 9_000, 0), (300, 24, 16, 8), (300, 24, 17, 9), (16, 129, 16, 1), (1, 7, 40_001, 0),                            # products of few rows
    (5, 64, 10_000, 3), (63, 30, 4_200, 8), (64, 30, 4_200, 8), (90, 30, 4_096, 8), (90, 30, 4_097, 9), (16_385, 8, 140, 8), (16_384, 8, 140, 8),   # losses with the teacher's scores
    (1_023, 16, 200, 8), (1_024, 16, 200, 8), (1_024, 16, 200, 9), (1_024, 16, 200, 32), (1_024, 16, 200, 33), (70, 16, 300, 129),                # the teacher's part of dz
])
def test_borders(torch, B, kind, n, D, C, k):
    check_all(torch, B, kind, inputs(torch, kind, n, D, C, k, seed=n + D + C + k), t=2.0, s=0.4 / n, st=0.6 / n)
