"""Orthogonalised updates by Newton-Schulz products.

Tolerance, in the norm of a matrix: X, A and the polynomial are rounded to binary16 in every step, half a
step of it is e = 2^-11 relative to a value; roundings of many values are independent, so the norm of their
sum is at most 0.58 of that (a uniform error) of each factor's norm.  In a step the polynomial's terms
reach |b| A + |c| A A < 4.8 + 2.1 while the result is at least 0.6 X, so a step adds at most
(4.8 + 2 * 2.1 + 3.5) * 0.58 e / 0.6 = 12 e, and less where it has not grown yet; later steps pass it on
with the polynomial's slope at the singular values near 1, at most 1.6 in magnitude over two steps and
below 1 on the average.  8 e bounds what is measured (5 e at the worst) and a product or layout gone
wrong is off by 0.1 or more.  The result's own rounding comes on top."""
import numpy as np
import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import CODES, HALF, TYPES, Placed, address, status, workspace

QUINTIC = (3.4445, -4.7750, 2.0315)


def plain(g, coefficients, eps, scale):
    x = g.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    turn = x.shape[-2] > x.shape[-1]
    x = x.transpose(-2, -1) if turn else x
    for a, b, c in coefficients:
        y = x @ x.transpose(-2, -1)
        x = a * x + (b * y + c * (y @ y)) @ x
    return scale * (x.transpose(-2, -1) if turn else x)


def test_the_formula_is_the_polynomial_of_the_singular_values():
    g = torch.Generator().manual_seed(1)
    for m, n in ((5, 8), (8, 5), (6, 6)):
        x = torch.randn(m, n, generator=g).double()
        u, s, v = torch.linalg.svd(x, full_matrices=False)
        s = s / x.norm()
        for _ in range(5):
            s = QUINTIC[0] * s + QUINTIC[1] * s ** 3 + QUINTIC[2] * s ** 5
        assert float((plain(x, [QUINTIC] * 5, 0.0, 1.0) - u @ torch.diag(s) @ v).norm()) < 1e-12
        assert 0.3 < float(s.min()) and float(s.max()) < 1.3


def test_refusals_need_no_gpu():
    keep, A = address()

    def f(g=A, dtype=nc.DTYPE_F32, batch=1, rows=8, cols=8, ldg=8, dist=64, co=QUINTIC, steps=1, eps=1e-7, out=A,
          ot=nc.DTYPE_BF16, ldo=8, od=64, ws=A, size=1 << 20):
        return nc.nc_orthogonalize(g, dtype, batch, rows, cols, ldg, dist, co, steps, eps, 1.0, out, ot, ldo,
                                   od, ws, size, stream=0)

    for kw in (dict(dtype=3), dict(ot=-1)):
        assert status(lambda: f(**kw)) == "NC_ERR_UNSUPPORTED", kw
    for kw in (dict(g=None), dict(out=None), dict(ws=None), dict(ldg=7), dict(ldo=7), dict(eps=-1.0),
               dict(eps=float("nan")), dict(batch=2, dist=63), dict(batch=2, od=63)):
        assert status(lambda: f(**kw)) == "NC_ERR_INVALID", kw
    for kw in (dict(g=A + 2), dict(out=A + 1), dict(ws=A + 16)):
        assert status(lambda: f(**kw)) == "NC_ERR_ALIGN", kw
    for kw in (dict(rows=(1 << 20) + 1), dict(cols=1 << 21, ldg=1 << 21, ldo=1 << 21), dict(batch=65536)):
        assert status(lambda: f(**kw)) == "NC_ERR_TOO_LARGE", kw
    assert status(lambda: f(size=100)) == "NC_ERR_WORKSPACE"
    assert status(lambda: f(co=QUINTIC * 1025, steps=1025)) == "NC_ERR_TOO_LARGE"
    for kw in (dict(batch=0), dict(rows=0), dict(cols=0)):
        assert status(lambda: f(**kw)) == "NC_OK", kw
    with pytest.raises(ValueError):
        f(steps=2)
    assert nc.nc_orthogonalize_workspace_bytes(1, 1 << 21, 8) == 0


def run(x, out="f32", coefficients=(QUINTIC,) * 5, eps=1e-7, scale=1.0, layout="whole", kind="f32"):
    batch, rows, cols = x.shape
    g, o = Placed(x.shape, kind, layout, x), Placed(x.shape, out, layout)
    size = nc.nc_orthogonalize_workspace_bytes(batch, rows, cols)
    memory, ws = workspace(size)
    nc.nc_orthogonalize(g.view, CODES[kind], batch, rows, cols, g.ld, g.distance,
                        [v for c in coefficients for v in c], len(coefficients), eps, scale, o.view,
                        CODES[out], o.ld, o.distance, ws, size)
    torch.cuda.synchronize()
    assert o.untouched() and bool((memory[:256] == 255).all()) and bool((memory[256 + size:] == 255).all())
    return g.view, o.view


def off(got, want):
    d = (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    return float(d.max())


SIZES = [(1, 1, 1), (3, 1, 70), (2, 33, 5), (2, 64, 64), (1, 255, 257), (2, 256, 512), (3, 300, 270), (1, 700, 64),
         (1, 1025, 513), (2, 40, 3000), (1, 2048, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols", SIZES)
def test_update(batch, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    for kind, out, layout in (("f32", "bf16", "whole"), ("bf16", "f32", "any"), ("f16", "f16", "gap"),
                              ("f32", "f32", "any"), ("f32", "f16", "gap")):
        x = 1e-3 * torch.randn(batch, rows, cols, generator=g, device="cuda")
        given, got = run(x, out, layout=layout, kind=kind, scale=1.5)
        want = plain(given, [tuple(float(np.float32(v)) for v in QUINTIC)] * 5, 1e-7, 1.5)
        assert off(got, want) <= 8 * 2.0 ** -11 + HALF[out], (kind, out, layout)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e25])
def test_any_size_of_the_gradient(size):
    x = size * torch.randn(1, 60, 90, device="cuda")
    given, got = run(x, eps=0.0)
    assert off(got, plain(given, [QUINTIC] * 5, 0.0, 1.0)) <= 8 * 2.0 ** -11


@pytest.mark.gpu
def test_low_rank_gradients():
    g = torch.Generator(device="cuda").manual_seed(5)
    for rows, cols in ((500, 700), (700, 500)):
        x = torch.randn(1, rows, 8, generator=g, device="cuda") @ torch.randn(1, 8, cols, generator=g, device="cuda")
        given, got = run(x)
        assert off(got, plain(given, [QUINTIC] * 5, 1e-7, 1.0)) <= 8 * 2.0 ** -11


@pytest.mark.gpu
def test_other_coefficients_and_no_steps():
    x = torch.randn(2, 100, 300, device="cuda")
    cubic = [(1.5, -0.5, 0.0)] * 9                     # converges to the orthogonal factor
    given, got = run(x, coefficients=cubic)
    assert off(got, plain(given, cubic, 1e-7, 1.0)) <= 8 * 2.0 ** -11
    many = [(1.0, -1e-3 * i, 1e-4) for i in range(35)]  # more than one launch takes, an odd number of X
    given, got = run(x, coefficients=many)
    assert off(got, plain(given, [tuple(float(np.float32(v)) for v in c) for c in many], 1e-7, 1.0)) <= 8 * 2.0 ** -11
    given, got = run(x, coefficients=(), scale=3.0)
    # X is kept in two binary16 values, 22 bits
    assert off(got, plain(given, [], 1e-7, 3.0)) <= 2.0 ** -20


@pytest.mark.gpu
def test_zeros_and_values_that_are_not_finite():
    x = torch.randn(4, 70, 50, device="cuda")
    x[1] = 0
    x[2, 3, 4] = float("nan")
    x[3, 69, 49] = float("inf")
    _, got = run(x, eps=0.0)
    assert bool(got[0].isfinite().all()) and bool((got[1] == 0).all())
    assert bool(got[2].isnan().all()) and bool(got[3].isnan().all())


@pytest.mark.gpu
def test_the_same_bits_captured_and_on_two_streams():
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(2, 300, 600, generator=g, device="cuda")
    size = nc.nc_orthogonalize_workspace_bytes(2, 300, 600)
    m = 300 * 600

    def call(out, ws):
        nc.nc_orthogonalize(x, nc.DTYPE_F32, 2, 300, 600, 600, m, QUINTIC * 5, 5, 1e-7, 1.0, out, nc.DTYPE_BF16,
                            600, m, ws, size)

    sets = [(torch.empty(2, 300, 600, dtype=torch.bfloat16, device="cuda"),
             torch.empty(size, dtype=torch.uint8, device="cuda")) for _ in range(4)]
    call(*sets[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, b in zip(streams, sets[1:3]):
            with torch.cuda.stream(s):
                call(*b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*sets[3])
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for b in sets[1:]:
        assert torch.equal(b[0], sets[0][0])
    x.copy_(x.flip(0))
    graph.replay()
    call(*sets[0])
    torch.cuda.synchronize()
    assert torch.equal(sets[3][0], sets[0][0])
