"""Orthogonalised updates at the ends of what the call accepts."""
import numpy as np
import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import HALF, address, status
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
@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 40), (1, 90)])
@pytest.mark.parametrize("co", [((2.0, 0.0, 0.0),) * 4, ((15.4, 0.0, 0.0), (0.5, -1.0, 0.0)), ((1.0, 0.0, 230.0),)])
def test_the_largest_coefficients_that_are_taken_overflow_nothing(co, rows, cols):
    # (a matrix of rank 1 has all of its norm in one singular value)
    x = torch.ones(1, rows, 1, device="cuda") @ torch.ones(1, 1, cols, device="cuda")
    x[0, 0, 0] += 1e-3
    for out in ("f32", "bf16"):
        given, got = run(x, out, coefficients=co)
        exact = [tuple(float(np.float32(v)) for v in c) for c in co]
        assert off(got, plain(given, exact, 1e-7, 1.0)) <= 8 * 2.0 ** -11 + HALF[out]


# ---- CPU: coefficients

def answer(coefficients):
    """What the call says to them, with a workspace of no bytes: it comes to that last."""
    keep, A = address()
    return status(lambda: nc.nc_orthogonalize(A, nc.DTYPE_F32, 1, 8, 8, 8, 64, [v for c in coefficients for v in c],
                                              len(coefficients), 1e-7, 1.0, A, nc.DTYPE_F32, 8, 64, A, 0, stream=0))


def largest(coefficients):
    """What the polynomials make of the singular values 0 to 1, and of their squares in b A + c A A, by trying:
    the largest squares and polynomials before a step."""
    s, worst = np.linspace(0, 1, 200001), 0.0
    for a, b, c in coefficients:
        u = s * s
        worst = np.max([worst, u.max(), np.abs(b * u + c * u * u).max()])      # (NaN stays NaN)
        s = np.linspace(0, np.abs(s * (a + b * u + c * u * u)).max(), 200001)
    return worst


TAKEN = [[QUINTIC] * 5, [QUINTIC] * 300, [(1.5, -0.5, 0.0)] * 40, [(2.0, 0.0, 0.0)] * 4, [(0.0, 0.0, 0.0)] * 3, [],
         [(1e30, -1e-30, 0.0)], [(8.287, -23.596, 17.3), (4.107, -2.948, 0.545), (3.949, -2.909, 0.552)],
         [(-2.0, 0.5, 0.0)] * 9, [(1.0, 200.0, -20.0)], [(0.0, -400.0, 400.0)]]
REFUSED = [[(2.0, 0.0, 0.0)] * 5, [(2.0, 0.0, 0.0)] * 10, [(1.0, 300.0, 0.0)], [(1.0, 0.0, -300.0)],
           [(16.0, 0.0, 0.0), (1.0, 0.0, 0.0)], [(1.0, 5.0, 5.0)] * 3, [(0.0, -1100.0, 1100.0)],
           [(0.0, -400.0, 400.0), (1.0, 0.0, 0.0)], [(float("nan"), 0.0, 0.0), (1.0, 0.0, 0.0)], [(1.0, float("nan"), 0.0)], [(1.0, 0.0, float("inf"))],
           [QUINTIC] * 20 + [(20.0, 0.0, 0.0)] + [QUINTIC]]


def test_coefficients_that_could_overflow_binary16_are_refused():
    for co in TAKEN:
        assert answer(co) == "NC_ERR_WORKSPACE", co[:3]
        assert largest(co) <= 240.0, co[:3]
    for co in REFUSED:
        assert answer(co) == "NC_ERR_INVALID", co[:3]
        assert not largest(co) <= 240.0, co[:3]


def test_coefficients_are_judged_by_the_values_that_they_reach():
    rng = np.random.default_rng(3)
    taken = 0
    for _ in range(300):
        co = [tuple(rng.normal(size=3) * rng.choice([1.0, 4.0, 30.0])) for _ in range(rng.integers(1, 5))]
        co = [tuple(float(np.float32(v)) for v in c) for c in co]
        worst = largest(co)
        if 239.9 < worst < 240.1:
            continue                      # (a grid of points is right to about 1e-9 of it)
        assert answer(co) == ("NC_ERR_WORKSPACE" if worst <= 240 else "NC_ERR_INVALID"), (co, worst)
        taken += worst <= 240
    assert 30 < taken < 270


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 2300, 2300), (5, 777, 1001), (40, 300, 290), (1, 2600, 4100)])
def test_more_tiles_than_pairs_of_blocks(batch, rows, cols):
    # a pair computes several tiles of a phase, whole ones and the narrow ones of the last round
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(batch, rows, cols, generator=g, device="cuda")
    for out, layout in (("f32", "any"), ("bf16", "whole")):
        given, got = run(x, out, layout=layout)
        exact = [tuple(float(np.float32(v)) for v in QUINTIC)] * 5
        assert off(got, plain(given, exact, 1e-7, 1.0)) <= 8 * 2.0 ** -11 + HALF[out]
