"""Orthogonalised updates at the ends of what the call accepts."""
import pytest
import torch

from operator_util import HALF
from test_orthogonalize import QUINTIC, off, plain, run


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [0, 1])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_matrix_that_is_not_finite_gives_nan_whatever_the_steps(bad, kind, steps):
    x = torch.randn(3, 70, 50, device="cuda")
    x[1, 3, 4] = bad
    _, got = run(x, kind=kind, coefficients=(QUINTIC,) * steps)
    assert bool(got[1].isnan().all())
    assert bool(got[0].isfinite().all()) and bool(got[2].isfinite().all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 40)])
def test_the_largest_coefficients_that_are_taken_overflow_nothing(rows, cols):
    # singular values of 1, 2, 4 and 8 before the steps of a matrix of rank 1, which has all of the norm in one
    x = torch.ones(1, rows, 1, device="cuda") @ torch.ones(1, 1, cols, device="cuda")
    x[0, 0, 0] += 1e-3
    for out in ("f32", "bf16"):
        given, got = run(x, out, coefficients=((2.0, 0.0, 0.0),) * 4)
        assert off(got, plain(given, [(2.0, 0.0, 0.0)] * 4, 1e-7, 1.0)) <= 8 * 2.0 ** -11 + HALF[out]
