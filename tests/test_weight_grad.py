"""Weight gradient of a linear layer whose input is kept as an 8-bit checkpoint.

Tolerances (u = 2^-24): the tensor cores add 16 products at a time to a binary32 sum and cut the
result off instead of rounding it, so a chain of rows / 16 steps is off by at most
(rows / 16 + 4) * 4 u times the sum of the terms' magnitudes (2 u for a cut, twice that for the sum
of 16 inside a step).  Column sums are rounded additions, at most rows of them.  The result is
rounded once to its type."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_1905_10988_b200 as nc
from test_act8_checkpoint import TYPES, _place, _status, matrix

U = 2.0 ** -24
ROUND = {"f32": U, "bf16": 2.0 ** -8}


# ---- CPU -----------------------------------------------------------------------------------

def test_plain_gradient_agrees_with_differences():
    rng = np.random.default_rng(2)
    t, n, k = 5, 3, 4
    xh, w, dy = rng.standard_normal((t, k)), rng.standard_normal((n, k)), rng.standard_normal((t, n))
    gamma, beta, bias = rng.standard_normal(k), rng.standard_normal(k), rng.standard_normal(n)
    dw, db = ref.weight_grad(dy, xh, gamma, beta)

    def loss(w, bias):
        return float((((xh * gamma + beta) @ w.T + bias) * dy).sum())

    h = 1e-6
    for i in range(n):
        e = np.zeros(n)
        e[i] = h
        assert abs((loss(w, bias + e) - loss(w, bias - e)) / (2 * h) - db[i]) < 1e-7
        for j in range(k):
            d = np.zeros((n, k))
            d[i, j] = h
            assert abs((loss(w + d, bias) - loss(w - d, bias)) / (2 * h) - dw[i, j]) < 1e-7


def test_workspace_holds_the_parts_of_a_split():
    # one tile of 256 x 256 and many tokens: split over the chip's pairs of blocks
    assert nc.nc_act8_weight_grad_workspace_bytes(1 << 16, 64, 64) >= 2 * 256 * 256 * 4
    assert nc.nc_act8_weight_grad_workspace_bytes(64, 256, 256) < 256 * 256 * 4
    assert nc.nc_act8_weight_grad_workspace_bytes(16384, 4096, 4096) < 1 << 26


def test_refusals_need_no_gpu():
    keep, A = _place()

    def f(dy=A, t=8, n=16, lddy=16, codes=A, scales=A, k=32, gamma=A, beta=A, pt=nc.DTYPE_F32, dw=A,
          wt=nc.DTYPE_BF16, lddw=32, db=A, ws=A, ws_bytes=1 << 20):
        return nc.nc_act8_weight_grad(dy, t, n, lddy, codes, scales, k, gamma, beta, pt, dw, wt,
                                      lddw, db, False, ws, ws_bytes, stream=0)

    assert _status(lambda: f(wt=nc.DTYPE_F16)) == "NC_ERR_UNSUPPORTED"
    assert _status(lambda: f(pt=9)) == "NC_ERR_UNSUPPORTED"
    for kw in (dict(dy=None), dict(lddy=15), dict(codes=None), dict(scales=None), dict(dw=None),
               dict(lddw=31), dict(ws=None)):
        assert _status(lambda: f(**kw)) == "NC_ERR_INVALID"
    for kw in (dict(dy=A + 1), dict(codes=A + 8), dict(scales=A + 8), dict(dw=A + 1),
               dict(db=A + 2), dict(gamma=A + 2), dict(beta=A + 2), dict(ws=A + 8),
               dict(wt=nc.DTYPE_F32, dw=A + 2)):
        assert _status(lambda: f(**kw)) == "NC_ERR_ALIGN"
    assert _status(lambda: f(ws_bytes=16)) == "NC_ERR_WORKSPACE"
    assert _status(lambda: f(t=1 << 31)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: f(n=1 << 31, lddy=1 << 31)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: f(k=1 << 31, lddw=1 << 31)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: f(n=1 << 21, lddy=1 << 21, k=1 << 21, lddw=1 << 21)) == "NC_ERR_TOO_LARGE"
    f(n=0)
    del keep


# ---- GPU ------------------------------------------------------------------------------------

def numpy64(t):
    return t.detach().cpu().double().numpy()


# one token, less than a step, a ragged step; sizes below, at and beyond half a tile and a tile;
# splits (long and narrow) and none; n of every alignment
SHAPES = [(1, 8, 32), (1, 1, 1), (17, 5, 40), (64, 128, 128), (65, 136, 160), (200, 256, 256),
          (513, 257, 300), (1000, 100, 513), (2048, 64, 64), (3000, 520, 264), (700, 1000, 1001)]


def run(t, n, k, affine, wkind, accumulate, dy_layout, dw_layout, seed=0, special=None):
    from gpu_util import Guarded
    rng = np.random.default_rng(seed + t + n + k)
    codes, scales = ref.encode(rng.standard_normal((t, k)).astype(np.float32)
                               * np.exp(rng.standard_normal((t, 1))).astype(np.float32))
    if special is not None:
        special(codes, scales)
    ldy, oy = {"whole": (n, 0), "gap": (-(-n // 8) * 8 + 8, 8), "any": (n + 3, 1)}[dy_layout]
    dy = matrix(t, n, ldy, oy, "bf16", torch.from_numpy(rng.standard_normal((t, n)) + 0.25))
    gamma = beta = None
    pkind = affine or "f32"
    if affine:
        gamma = torch.from_numpy(rng.standard_normal(k)).cuda().to(TYPES[pkind][1])
        beta = torch.from_numpy(rng.standard_normal(k)).cuda().to(TYPES[pkind][1])
    ldw, ow = {"whole": (k, 0), "any": (k + 5, 1)}[dw_layout]
    dw = matrix(n, k, ldw, ow, wkind)
    old = torch.from_numpy(rng.standard_normal((n, k))).to(TYPES[wkind][1])
    dw.copy_(old if accumulate else torch.full_like(old, 7.0))
    db = Guarded(4 * n)
    oldb = rng.standard_normal(n).astype(np.float32)
    db.buf.copy_(torch.from_numpy(oldb.view(np.uint8)))
    ws_bytes = nc.nc_act8_weight_grad_workspace_bytes(t, n, k)
    ws = Guarded(ws_bytes)
    c, s = Guarded(nc.nc_act8_code_bytes(t, k)), Guarded(nc.nc_act8_scale_bytes(t, k))
    c.buf.copy_(torch.from_numpy(codes.reshape(-1)))
    s.buf[:scales.size].copy_(torch.from_numpy(scales.reshape(-1)))
    nc.nc_act8_weight_grad(dy, t, n, ldy, c.buf, s.buf, k, gamma, beta, TYPES[pkind][0], dw,
                           TYPES[wkind][0], ldw, db.buf, accumulate, ws.buf, ws_bytes)
    torch.cuda.synchronize()
    for b in (ws, db, c, s):
        b.check()
    store = torch.empty(0, dtype=dw.dtype, device="cuda").set_(dw.untyped_storage())
    mask = torch.ones_like(store, dtype=torch.bool)
    mask[ow:ow + n * ldw].view(n, ldw)[:, :k] = False
    assert not bool(store[mask].float().ne(0).any()), "write outside the rows"
    xh = ref.decode(codes, scales, k)
    d64 = numpy64(dy)
    g64 = numpy64(gamma) if affine else None
    b64 = numpy64(beta) if affine else None
    want, wantb = ref.weight_grad(d64, xh, g64, b64)
    terms = np.abs(d64).T @ np.abs(xh)
    tol = (t / 16 + 4) * 4 * U * terms
    sums = np.abs(d64).sum(0)
    tolb = (t + 4) * U * sums
    if affine:
        tol = tol * np.abs(g64) + np.outer(tolb, np.abs(b64)) + 4 * U * (
            terms * np.abs(g64) + np.outer(sums, np.abs(b64)))
    if accumulate:
        want, wantb = want + numpy64(old), wantb + oldb
        tol, tolb = tol + U * np.abs(want), tolb + U * np.abs(wantb)
    tol = tol + ROUND[wkind] * (np.abs(want) + tol) + 2.0 ** -134
    return numpy64(dw), want, tol, db.numpy(np.float32), wantb, tolb


@pytest.mark.gpu
@pytest.mark.parametrize("t,n,k", SHAPES)
@pytest.mark.parametrize("dy_layout,dw_layout", [("whole", "whole"), ("gap", "any"),
                                                 ("any", "whole")])
@pytest.mark.parametrize("affine,wkind,accumulate", [(None, "bf16", False), ("bf16", "f32", False),
                                                     ("f32", "bf16", True), ("f16", "f32", True)])
def test_gpu_weight_gradient(t, n, k, dy_layout, dw_layout, affine, wkind, accumulate):
    got, want, tol, gotb, wantb, tolb = run(t, n, k, affine, wkind, accumulate, dy_layout,
                                            dw_layout)
    assert np.all(np.abs(got - want) <= tol), np.abs(got - want).max()
    assert np.all(np.abs(gotb - wantb) <= tolb)


@pytest.mark.gpu
@pytest.mark.parametrize("t,n,k,dy_layout", [(130, 5128, 2100, "whole"), (70, 5299, 2050, "any"),
                                             (200, 9000, 2304, "gap"), (65, 5128, 2100, "any")])
def test_gpu_more_tiles_than_pairs(t, n, k, dy_layout):
    # rounds of double tiles, then single ones, then a rest; an odd number of tiles along n
    got, want, tol, gotb, wantb, tolb = run(t, n, k, "bf16", "bf16", False, dy_layout, "whole")
    assert np.all(np.abs(got - want) <= tol)
    assert np.all(np.abs(gotb - wantb) <= tolb)


@pytest.mark.gpu
def test_gpu_long_contraction():
    got, want, tol, gotb, wantb, tolb = run(20_000, 300, 700, "bf16", "f32", False, "whole",
                                            "whole")
    assert np.all(np.abs(got - want) <= tol)
    assert np.all(np.abs(gotb - wantb) <= tolb)


@pytest.mark.gpu
def test_gpu_every_scale_and_a_block_that_is_not_finite():
    # all scale bytes that the tensor cores' operand can hold: from 2^-118 to 2^112 (a product of
    # 127 * 2^112 and dy stays finite)
    def scales_of(codes, scales):
        scales[:, :] = (9 + np.arange(scales.size) * 7 % 231).reshape(scales.shape).astype(np.uint8)
        scales[5] = 9
    got, want, tol, _, _, _ = run(160, 64, 96, None, "f32", False, "whole", "whole",
                                  special=scales_of)
    assert np.all(np.abs(got - want) <= tol)

    def broken(codes, scales):
        scales[3, 1] = 255
        codes[3, 32:64] = 0
    got, want, _, _, _, _ = run(70, 20, 96, None, "f32", False, "whole", "whole", special=broken)
    assert np.isnan(got[:, 32:64]).all() and np.isfinite(got[:, :32]).all()
    assert np.isfinite(got[:, 64:]).all()


@pytest.mark.gpu
def test_gpu_large_units_take_the_slow_decoder():
    def large(codes, scales):
        scales[:, :] = 127
        scales[7, 0] = 248                  # 2^121: one value a row of codes, dy of the row tiny
        codes[7, :32] = 0
        codes[7, 4] = 1
    got, want, tol, _, _, _ = run(40, 16, 32, None, "f32", False, "whole", "whole", special=large)
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.gpu
def test_gpu_no_tokens_no_columns():
    dw = torch.full((3, 5), 2.0, device="cuda")
    db = torch.full((3,), 4.0, device="cuda")
    F = nc.DTYPE_F32

    def call(k, accumulate):
        nc.nc_act8_weight_grad(None, 0, 3, 3, None, None, k, None, None, F, dw, F, 5, db, accumulate,
                               None, 0)

    call(5, True)
    assert bool((dw == 2).all()) and bool((db == 4).all())
    call(0, False)
    assert bool((dw == 2).all()) and not bool(db.any())
    call(5, False)
    assert not bool(dw.any())


@pytest.mark.gpu
def test_gpu_repeatable_and_on_another_stream():
    t, n, k = 4096, 256, 320
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn(t, n, generator=g, device="cuda").bfloat16()
    x = torch.randn(t, k, generator=g, device="cuda")
    u8 = dict(dtype=torch.uint8, device="cuda")
    codes = torch.empty(nc.nc_act8_code_bytes(t, k), **u8)
    scales = torch.empty(nc.nc_act8_scale_bytes(t, k), **u8)
    nc.nc_act8_compress(x, nc.DTYPE_F32, t, k, k, nc.ROUND_NEAREST, 0, 0, codes, scales)
    b = nc.nc_act8_weight_grad_workspace_bytes(t, n, k)
    outs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side, None):
        dw, db = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
        ws = torch.empty(b, **u8)
        torch.cuda.synchronize()
        nc.nc_act8_weight_grad(dy, t, n, n, codes, scales, k, None, None, nc.DTYPE_F32, dw,
                               nc.DTYPE_F32, k, db, False, ws, b, stream=stream)
        torch.cuda.synchronize()
        outs.append((dw, db))
    for o in outs[1:]:
        assert all(torch.equal(p, q) for p, q in zip(o, outs[0]))


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [False, True])
def test_gpu_no_tokens_give_zero_whatever_the_parameters_are(accumulate):
    # a sum over no tokens has no term that an inf or NaN parameter could reach
    dw = torch.full((3, 40), 2.0, device="cuda")
    db = torch.full((3,), 4.0, device="cuda")
    gamma = torch.full((40,), float("inf"), device="cuda")
    beta = torch.full((40,), float("nan"), device="cuda")
    F = nc.DTYPE_F32
    nc.nc_act8_weight_grad(None, 0, 3, 3, None, None, 40, gamma, beta, F, dw, F, 40, db, accumulate,
                           None, 0)
    assert bool((dw == (2 if accumulate else 0)).all()) and bool((db == (4 if accumulate else 0)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("wkind,tokens", [("f32", 8192), ("bf16", 16384)])
def test_gpu_error_does_not_grow_with_the_number_of_tokens(wkind, tokens):
    # An accumulator cuts off at most an ulp, 2^-23 of its value, each time 16 tokens are added, and is
    # emptied after `tokens` at most.  The sums of terms of either sign grow like the square root of
    # their number, so a chain of m additions loses at most 2^-23 * sum of sqrt(s / m) = 2/3 m 2^-23 of
    # its value, and the sum of chains as much of theirs; rounding adds u for every chain and the
    # result's own rounding, which is as often up as down.
    t, n, k = 1 << 18, 2560, 2048                     # more tiles than pairs: whole ones and split ones
    g = torch.Generator(device="cuda").manual_seed(3)
    u8 = dict(dtype=torch.uint8, device="cuda")
    dy = torch.randn(t, n, generator=g, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(t, k, generator=g, device="cuda", dtype=torch.bfloat16)
    codes = torch.empty(nc.nc_act8_code_bytes(t, k), **u8)
    scales = torch.empty(nc.nc_act8_scale_bytes(t, k), **u8)
    B = nc.DTYPE_BF16
    nc.nc_act8_compress(x, B, t, k, k, nc.ROUND_NEAREST, 0, 0, codes, scales)
    nc.nc_act8_decompress(codes, scales, t, k, x, B, k)            # exact
    size = nc.nc_act8_weight_grad_workspace_bytes(t, n, k)
    ws = torch.empty(size, **u8)
    dw = torch.empty(n, k, device="cuda", dtype=TYPES[wkind][1])
    nc.nc_act8_weight_grad(dy, t, n, n, codes, scales, k, None, None, nc.DTYPE_F32, dw,
                           TYPES[wkind][0], k, None, False, ws, size)
    want = torch.zeros(n, k, dtype=torch.float64, device="cuda")
    for i in range(0, t, 16384):
        want += dy[i:i + 16384].double().t() @ x[i:i + 16384].double()
    err = dw.double() - want
    bound = 2 / 3 * (tokens / 16) * 2.0 ** -23 + (t / tokens + 2) * U
    if wkind == "f32":
        assert float(err.norm() / want.norm()) <= bound
    # towards 0 by so much of the value; rounding to bfloat16 averages out over the entries
    toward = float((err * want.sign()).sum() / want.abs().sum())
    assert abs(toward) <= bound + 4 * ROUND[wkind] / (n * k) ** 0.5


# ---- the schedule that large layers take -------------------------------------------------------

PAIRS, TILE, STEP = 74, 256, 64


def plan(t, n, k):
    """rounds of double tiles, rounds of whole single ones, tiles left over and their parts, where dY
    comes by tensor copies"""
    tn, tk, steps = -(-n // TILE), -(-k // TILE), -(-t // STEP)
    doubles = tn // 2 * tk // PAIRS
    tiles = tn * tk - 2 * PAIRS * doubles
    left = tiles % PAIRS
    splits = max(1, min(PAIRS // left if left else 1, steps // 4))
    return doubles, tiles // PAIRS, left, splits


# (what the shape is for, tokens, n, k, layout of dY, affine, type of dW, accumulate)
LARGE = [("single tiles one after another", 130, 4096, 2048, "whole", "f32", "f32", True),
         ("double, single and split ones", 600, 4096, 4096, "whole", "bf16", "bf16", True),
         ("the same through the aligned copy", 600, 4095, 4096, "whole", "f16", "f32", False),
         ("the same with gaps, a ragged last step", 577, 4000, 4090, "gap", "f32", "f32", True)]


def test_large_shapes_take_the_paths_that_they_are_for():
    # (doubles, rounds of whole ones, left over, parts)
    assert [plan(*c[1:4]) for c in LARGE] == [(0, 1, 54, 1), (1, 1, 34, 2), (1, 1, 34, 2), (1, 1, 34, 2)]
    assert LARGE[2][2] % 8 and not LARGE[3][2] % 8


@pytest.mark.gpu
@pytest.mark.parametrize("case", LARGE, ids=[c[0] for c in LARGE])
def test_gpu_schedule_of_large_layers(case):
    _, t, n, k, layout, affine, wkind, accumulate = case
    got, want, tol, gotb, wantb, tolb = run(t, n, k, affine, wkind, accumulate, layout, "whole")
    assert np.all(np.abs(got - want) <= tol), np.abs(got - want).max()
    assert np.all(np.abs(gotb - wantb) <= tolb)


@pytest.mark.gpu
def test_gpu_every_scale_byte_at_its_own_magnitude():
    # a block of 32 columns has one scale byte in every row, so that each byte is seen in results of its
    # own size; products below 2^-126 may be taken for 0
    count, t = 231, 48

    def scales_of(codes, scales):
        scales[:, :] = 9 + np.arange(count, dtype=np.uint8)

    got, want, tol, _, _, _ = run(t, 16, 32 * count, None, "f32", False, "whole", "whole",
                                  special=scales_of)
    assert np.all(np.abs(got - want) <= tol + t * 2.0 ** -126)
    # and the tolerance tells a byte from its neighbours
    assert np.all(np.median(np.abs(want) / (tol + t * 2.0 ** -126), axis=0) > 100)
