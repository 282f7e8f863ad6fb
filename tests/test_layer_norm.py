"""Layer norm forward and backward, from the saved input and from the 8-bit checkpoint: the plain
64-bit form against differences on CPU, refusals, and the CUDA path against the plain form.

Tolerances (u = 2^-24, t = unit roundoff of the output type): a binary32 sum of n terms in the
kernels is a serial chain of at most 32 terms a thread, 5 shuffle steps and at most 64 warps, so
it is off by at most 101 u times the sum of the terms' magnitudes; parameter gradients have a
chain of the rows of an owner and of the owners' parts instead.  Every other operation adds one u
of its result."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_1905_10988_b200 as nc
from test_act8_checkpoint import TYPES, _place, _status, matrix

U = 2.0 ** -24
CHAIN = 101
ROUND = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}   # half a subnormal step
EPS = 1e-5


# ---- CPU -----------------------------------------------------------------------------------

def test_plain_gradient_agrees_with_differences():
    rng = np.random.default_rng(1)
    rows, cols = 3, 7
    x = rng.standard_normal((rows, cols))
    gamma, beta = rng.standard_normal(cols), rng.standard_normal(cols)
    w = rng.standard_normal((rows, cols))
    _, _, rstd, xh = ref.layer_norm(x, gamma, beta, EPS)
    dx, dgamma, dbeta = ref.layer_norm_backward(w, xh, rstd, gamma)

    def loss(x, gamma, beta):
        return float((ref.layer_norm(x, gamma, beta, EPS)[0] * w).sum())

    h = 1e-6
    for i in range(rows):
        for j in range(cols):
            d = np.zeros_like(x)
            d[i, j] = h
            num = (loss(x + d, gamma, beta) - loss(x - d, gamma, beta)) / (2 * h)
            assert abs(num - dx[i, j]) < 1e-7
    for j in range(cols):
        d = np.zeros(cols)
        d[j] = h
        assert abs((loss(x, gamma + d, beta) - loss(x, gamma - d, beta)) / (2 * h) - dgamma[j]) < 1e-7
        assert abs((loss(x, gamma, beta + d) - loss(x, gamma, beta - d)) / (2 * h) - dbeta[j]) < 1e-7


def test_refusals_need_no_gpu():
    keep, A = _place()

    def fwd(x=A, dt=nc.DTYPE_BF16, r=4, c=40, ldx=40, gamma=A, beta=A, pt=nc.DTYPE_F32, y=A,
            ldy=40, mean=A, rstd=A, codes=A, scales=A, mode=0):
        return nc.nc_layer_norm_forward(x, dt, r, c, ldx, gamma, beta, pt, EPS, y, ldy, mean, rstd,
                                        codes, scales, mode, 0, 0, stream=0)

    ws = 1 << 20

    def bwd(dy=A, dt=nc.DTYPE_BF16, r=4, c=40, lddy=40, x=A, ldx=40, mean=A, rstd=A, gamma=A,
            pt=nc.DTYPE_F32, dres=None, lddres=0, dx=A, lddx=40, dgamma=A, dbeta=A, workspace=A,
            ws=ws):
        return nc.nc_layer_norm_backward(dy, dt, r, c, lddy, x, ldx, mean, rstd, gamma, pt, dres,
                                         lddres, dx, lddx, dgamma, dbeta, False, workspace, ws,
                                         stream=0)

    def bwd8(dy=A, dt=nc.DTYPE_BF16, r=4, c=40, lddy=40, codes=A, scales=A, rstd=A, gamma=A,
             pt=nc.DTYPE_F32, dres=None, lddres=0, dx=A, lddx=40, dgamma=A, dbeta=A, workspace=A,
             ws=ws):
        return nc.nc_act8_layer_norm_backward(dy, dt, r, c, lddy, codes, scales, rstd, gamma, pt,
                                              dres, lddres, dx, lddx, dgamma, dbeta, False,
                                              workspace, ws, stream=0)

    for f in (fwd, bwd, bwd8):
        assert _status(lambda: f(dt=7)) == "NC_ERR_UNSUPPORTED"
        assert _status(lambda: f(pt=-1)) == "NC_ERR_UNSUPPORTED"
        assert _status(lambda: f(rstd=A + 2)) == "NC_ERR_ALIGN"
        assert _status(lambda: f(gamma=A + 2)) == "NC_ERR_ALIGN"
        f(c=0)
    wide = dict(c=32769)
    assert _status(lambda: fwd(ldx=32769, ldy=32769, **wide)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: bwd(lddy=32769, ldx=32769, lddx=32769, **wide)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: bwd8(lddy=32769, lddx=32769, **wide)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: fwd(r=1 << 31)) == "NC_ERR_TOO_LARGE"
    assert _status(lambda: bwd(r=1 << 31)) == "NC_ERR_TOO_LARGE"
    fwd(r=0)
    for kw in (dict(x=None), dict(y=None), dict(ldx=39), dict(ldy=39), dict(scales=None),
               dict(codes=None), dict(mode=5)):
        assert _status(lambda: fwd(**kw)) == "NC_ERR_INVALID"
    assert _status(lambda: fwd(codes=A + 1)) == "NC_ERR_ALIGN"
    assert _status(lambda: fwd(y=A + 1)) == "NC_ERR_ALIGN"
    for f in (bwd, bwd8):
        for kw in (dict(dy=None), dict(dx=None), dict(rstd=None), dict(dgamma=None),
                   dict(dbeta=None), dict(lddy=39), dict(lddx=39), dict(workspace=None),
                   dict(dres=A, lddres=39)):
            assert _status(lambda: f(**kw)) == "NC_ERR_INVALID"
        assert _status(lambda: f(ws=16)) == "NC_ERR_WORKSPACE"
        assert _status(lambda: f(workspace=A + 4)) == "NC_ERR_ALIGN"
        assert _status(lambda: f(dgamma=A + 2)) == "NC_ERR_ALIGN"
        assert _status(lambda: f(dres=A + 1, lddres=40)) == "NC_ERR_ALIGN"
    assert _status(lambda: bwd(x=None)) == "NC_ERR_INVALID"
    assert _status(lambda: bwd(mean=None)) == "NC_ERR_INVALID"
    assert _status(lambda: bwd(ldx=39)) == "NC_ERR_INVALID"
    assert _status(lambda: bwd8(codes=None)) == "NC_ERR_INVALID"
    assert _status(lambda: bwd8(scales=None)) == "NC_ERR_INVALID"
    assert _status(lambda: bwd8(codes=A + 8)) == "NC_ERR_ALIGN"
    del keep


def test_workspace_size():
    assert nc.nc_layer_norm_workspace_bytes(0, 64) == 0
    assert nc.nc_layer_norm_workspace_bytes(1, 33) == 2 * 64 * 4
    assert nc.nc_layer_norm_workspace_bytes(10 ** 6, 4096) <= 592 * 2 * 4096 * 4


def test_workspace_of_no_columns():
    # asked for before a call that has nothing to do; in a process of its own, which a division by
    # zero in the library would end
    code = ("import paper_1905_10988_b200 as nc\n"
            "assert nc.nc_layer_norm_workspace_bytes(4, 0) == 0\n"
            "assert nc.nc_layer_norm_workspace_bytes(0, 0) == 0\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run([sys.executable, "-c", code], cwd=root).returncode == 0


# ---- GPU ------------------------------------------------------------------------------------

def numpy64(t):
    return t.detach().cpu().double().numpy()


def rows_of(rng, rows, cols):
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))
    return x + 3.0 * rng.standard_normal((rows, 1))


# every assignment of a row to threads: a warp (1 or 2 chunks), a block, a block with 2 chunks or a
# cluster of 2 or 4 blocks; one row, ragged widths, fewer and more rows than owners
SHAPES = [(1, 1), (1, 5), (3, 32), (5, 512), (9, 513), (4, 1000), (70, 1024), (2, 1025),
          (700, 2000), (3, 4096), (5, 8192), (3, 8193), (2, 16384), (3, 16400), (2, 32768),
          (2500, 96)]
LAYOUTS = ["whole", "gap16", "any"]


def layout(name, cols, size):
    """row stride and offset in elements"""
    if name == "whole":
        return cols, 0
    if name == "gap16":                       # rows on 16-byte boundaries, some not on 32
        return -(-cols // 8) * 8 + 16 // size + (8 if size == 2 else 4), 16 // size
    if name == "gap32":                       # rows on 32-byte boundaries
        return cols + 32 // size, 32 // size
    return cols + 1, 1


@pytest.mark.gpu
@pytest.mark.parametrize("kind,pkind", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                        ("f16", "f16")])
@pytest.mark.parametrize("where", LAYOUTS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gpu_forward(kind, pkind, where, rows, cols):
    from gpu_util import Guarded
    rng = np.random.default_rng(rows + cols)
    code, dt = TYPES[kind]
    ld, off = layout(where, cols, 4 if kind == "f32" else 2)
    x = matrix(rows, cols, ld, off, kind, torch.from_numpy(rows_of(rng, rows, cols)).cuda())
    y = matrix(rows, cols, ld, off, kind)
    gamma = torch.from_numpy(rng.standard_normal(cols)).cuda().to(TYPES[pkind][1])
    beta = torch.from_numpy(rng.standard_normal(cols)).cuda().to(TYPES[pkind][1])
    mean, rstd = Guarded(4 * rows), Guarded(4 * rows)
    x64 = numpy64(x)
    wy, wmean, wrstd, wxh = ref.layer_norm(x64, numpy64(gamma), numpy64(beta), EPS)
    # error of the mean, of a centred value, and of xh (the rstd: half that of the variance, whose
    # terms carry twice the relative error of a centred value)
    emean = (CHAIN + 2) * U * np.abs(x64).mean(1)
    centred = np.abs(x64 - wmean[:, None])
    ecent = emean[:, None] + U * (centred + emean[:, None])
    evar = (2 * centred * ecent + ecent ** 2).mean(1) + (CHAIN + 3) * U * (centred ** 2).mean(1)
    erstd = wrstd * (0.51 * evar * wrstd ** 2 + 4 * U)
    exh = ecent * (wrstd + erstd)[:, None] + centred * erstd[:, None] + U * np.abs(wxh)
    g64, b64 = np.abs(numpy64(gamma)), np.abs(numpy64(beta))
    ey = exh * g64 + 2 * U * (np.abs(wxh) * g64 + b64)
    ey = ey + ROUND[kind] * (np.abs(wy) + ey) + SMALLEST[kind]
    for keep in (None, "nearest", "random"):
        codes = scales = None
        if keep:
            codes = Guarded(nc.nc_act8_code_bytes(rows, cols))
            scales = Guarded(nc.nc_act8_scale_bytes(rows, cols))
        mode = nc.ROUND_RANDOM if keep == "random" else nc.ROUND_NEAREST
        y.zero_()
        nc.nc_layer_norm_forward(x, code, rows, cols, ld, gamma, beta, TYPES[pkind][0], EPS, y, ld,
                                 mean.buf, rstd.buf, codes.buf if keep else None,
                                 scales.buf if keep else None, mode, 77, 2)
        torch.cuda.synchronize()
        for b in (mean, rstd, codes, scales):
            if b is not None:
                b.check()
        assert np.all(np.abs(mean.numpy(np.float32) - wmean) <= emean + U * np.abs(wmean) + 1e-45)
        assert np.all(np.abs(rstd.numpy(np.float32) - wrstd) <= erstd)
        assert np.all(np.abs(numpy64(y) - wy) <= ey)
        if not keep:
            continue
        # the unit of every block is that of its largest |xh|, or a neighbour's where the error of
        # xh crosses the boundary; a value is off by half a unit (nearest) or by less than one
        # unit and the half 1/256 of the draws' grid (random)
        p = ref.pitch_of(cols)
        c = codes.numpy(np.uint8).reshape(rows, p)
        s = scales.numpy(np.uint8)[:rows * p // 32].reshape(rows, p // 32)
        lo, hi = np.abs(wxh) - exh, np.abs(wxh) + exh
        assert np.all(s >= ref.scale_bytes(np.maximum(lo, 0)))
        assert np.all(s <= ref.scale_bytes(hi))
        unit = np.ldexp(1.0, np.repeat(s.astype(int), 32, 1)[:, :cols] - 127)
        off_by = np.abs(ref.decode(c, s, cols) - wxh)
        part = 0.5 if keep == "nearest" else 1.0 + 1.0 / 512
        assert np.all(off_by <= part * unit + exh)
        assert not c[:, cols:].any()
        if keep == "random":
            # rounded with the documented draws: the value lies above xh by its draw at most
            r = ref.stream_bytes(77, 2, rows * p).reshape(rows, p)[:, :cols].astype(np.float64)
            m = (c[:, :cols] & 127).astype(np.float64)
            fine = np.abs(wxh) / unit * 256
            tol = exh / unit * 256 + 0.5
            assert np.all(m * 256 <= fine + r + tol) and np.all(m * 256 + 255 >= fine + r - tol)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,pkind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("where", LAYOUTS)
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("saved8", [False, True])
def test_gpu_backward(kind, pkind, where, rows, cols, saved8):
    from gpu_util import Guarded
    rng = np.random.default_rng(rows + 3 * cols)
    code, dt = TYPES[kind]
    ld, off = layout(where, cols, 4 if kind == "f32" else 2)
    x = matrix(rows, cols, ld, off, kind, torch.from_numpy(rows_of(rng, rows, cols)).cuda())
    dy = matrix(rows, cols, ld, off, kind, torch.from_numpy(rng.standard_normal((rows, cols)) + 0.3))
    dres = matrix(rows, cols, ld, off, kind, torch.from_numpy(rng.standard_normal((rows, cols))))
    gamma = torch.from_numpy(rng.standard_normal(cols)).cuda().to(TYPES[pkind][1])
    _, m64, r64, xh64 = ref.layer_norm(numpy64(x), None, None, EPS)
    mean = torch.from_numpy(m64.astype(np.float32)).cuda()
    rstd = torch.from_numpy(r64.astype(np.float32)).cuda()
    if saved8:
        c, s = ref.encode(xh64.astype(np.float32))
        codes, scales = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
        xh, exh = ref.decode(c, s, cols), 0.0
    else:
        xh = (numpy64(x) - numpy64(mean)[:, None]) * numpy64(rstd)[:, None]
        exh = 2.1 * U * np.abs(xh)
    ws_bytes = nc.nc_layer_norm_workspace_bytes(rows, cols)
    ws, dgamma, dbeta = Guarded(ws_bytes), Guarded(4 * cols), Guarded(4 * cols)
    dx = matrix(rows, cols, ld, off, kind)
    chain = min(rows, 130 + rows // 100) + 90          # rows of an owner, its warps, 592 / 8 parts
    old = rng.standard_normal(cols).astype(np.float32)
    for with_gamma, with_res, accumulate in [(True, False, False), (False, True, True),
                                             (True, True, False)]:
        gm = gamma if with_gamma else None
        dr = dres if with_res else None
        if accumulate:
            for b in (dgamma, dbeta):
                b.buf.copy_(torch.from_numpy(old.view(np.uint8)).cuda())
        dx.zero_()
        tail = (TYPES[pkind][0], dr, ld, dx, ld, dgamma.buf, dbeta.buf, accumulate, ws.buf, ws_bytes)
        if saved8:
            nc.nc_act8_layer_norm_backward(dy, code, rows, cols, ld, codes, scales, rstd, gm, *tail)
        else:
            nc.nc_layer_norm_backward(dy, code, rows, cols, ld, x, ld, mean, rstd, gm, *tail)
        torch.cuda.synchronize()
        for b in (ws, dgamma, dbeta):
            b.check()
        g64 = numpy64(gamma) if with_gamma else None
        wdx, wdg, wdb = ref.layer_norm_backward(numpy64(dy), xh, numpy64(rstd), g64,
                                                numpy64(dres) if with_res else None)
        g = numpy64(dy) * (1.0 if g64 is None else g64)
        ag, ax = np.abs(g), np.abs(xh)
        m1, m2 = ag.mean(1, keepdims=True), (ag * ax).mean(1, keepdims=True)
        e1 = (CHAIN + 3) * U * m1
        e2 = (CHAIN + 4) * U * m2 + (ag * exh).mean(1, keepdims=True)
        inner = ag + m1 + ax * m2
        e = np.abs(numpy64(rstd))[:, None] * (e1 + ax * e2 + (exh + U * ax) * m2 + 5 * U * inner)
        if with_res:
            e = e + U * (np.abs(wdx) + np.abs(numpy64(dres)))
        e = e + ROUND[kind] * (np.abs(wdx) + e) + SMALLEST[kind]
        assert np.all(np.abs(numpy64(dx) - wdx) <= e)
        ady = np.abs(numpy64(dy))
        base = old.astype(np.float64) if accumulate else 0.0
        tg = (chain + 2) * U * (ady * ax).sum(0) + (ady * exh).sum(0) + U * np.abs(base + wdg)
        tb = (chain + 1) * U * ady.sum(0) + U * np.abs(base + wdb)
        assert np.all(np.abs(dgamma.numpy(np.float32) - (base + wdg)) <= tg + 1e-45)
        assert np.all(np.abs(dbeta.numpy(np.float32) - (base + wdb)) <= tb + 1e-45)


# several rows an owner: rows whose values fill every thread (32 a thread forward; backward through
# the ring, which comes round), of a warp, a block or a cluster, and such that do not
MANY = [(5000, 512), (2500, 1024), (520, 2048), (1300, 4096), (600, 5120), (700, 7168), (700, 8192),
        (513, 8200), (1500, 1001), (700, 4099)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,pkind,where", [("f32", "f32", "gap32"), ("bf16", "bf16", "whole"),
                                              ("f16", "f32", "gap32")])
@pytest.mark.parametrize("rows,cols", MANY)
def test_gpu_forward_many_rows(kind, pkind, where, rows, cols):
    test_gpu_forward(kind, pkind, where, rows, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,pkind,where", [("f32", "f32", "gap32"), ("bf16", "bf16", "whole"),
                                              ("f16", "f32", "gap32")])
@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("saved8", [False, True])
def test_gpu_backward_many_rows(kind, pkind, where, rows, cols, saved8):
    test_gpu_backward(kind, pkind, where, rows, cols, saved8)


@pytest.mark.gpu
def test_gpu_gradient_agrees_with_differences_of_the_forward():
    # central differences of sum(w * layer_norm(x)) in float64 at the binary32 inputs
    rng = np.random.default_rng(8)
    rows, cols = 4, 50
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    w = rng.standard_normal((rows, cols)).astype(np.float32)
    gamma = rng.standard_normal(cols).astype(np.float32)
    xd, wd, gd = (torch.from_numpy(a).cuda() for a in (x, w, gamma))
    y, dx = torch.empty_like(xd), torch.empty_like(xd)
    f32 = dict(dtype=torch.float32, device="cuda")
    mean, rstd = torch.empty(rows, **f32), torch.empty(rows, **f32)
    dgamma, dbeta = torch.empty(cols, **f32), torch.empty(cols, **f32)
    n = nc.nc_layer_norm_workspace_bytes(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    F = nc.DTYPE_F32
    nc.nc_layer_norm_forward(xd, F, rows, cols, cols, gd, None, F, EPS, y, cols, mean, rstd, None,
                             None, 0, 0, 0)
    nc.nc_layer_norm_backward(wd, F, rows, cols, cols, xd, cols, mean, rstd, gd, F, None, 0, dx,
                              cols, dgamma, dbeta, False, ws, n)
    h = 1e-5
    got = dx.cpu().numpy()
    for i in range(rows):
        for j in range(cols):
            d = np.zeros((rows, cols))
            d[i, j] = h
            a = (ref.layer_norm(x + d, gamma, None, EPS)[0] * w).sum()
            b = (ref.layer_norm(x - d, gamma, None, EPS)[0] * w).sum()
            # differences: O(h^2) and rounding / h; the kernel: a few hundred u of terms below 30
            assert abs((a - b) / (2 * h) - got[i, j]) < 1e-6 + 500 * U * 30


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [40, 2000, 20000])
def test_gpu_rows_that_are_not_finite_stay_by_themselves(cols):
    rows = 5
    x = torch.randn(rows, cols, device="cuda")
    x[1, cols // 2] = float("inf")
    x[3, 0] = float("nan")
    y = torch.empty_like(x)
    rstd = torch.empty(rows, device="cuda")
    codes = torch.empty(nc.nc_act8_code_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    scales = torch.empty(nc.nc_act8_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    F = nc.DTYPE_F32
    nc.nc_layer_norm_forward(x, F, rows, cols, cols, None, None, F, EPS, y, cols, None, rstd,
                             codes, scales, 0, 0, 0)
    back = torch.empty_like(x)
    nc.nc_act8_decompress(codes, scales, rows, cols, back, F, cols)
    for t in (y, back):
        bad = ~torch.isfinite(t)
        assert bool(bad[1].all()) and bool(bad[3].all())
        assert not bool(bad[[0, 2, 4]].any())
    # the gradient of a row with NaN is NaN in dx there, and in the sums over rows
    n = nc.nc_layer_norm_workspace_bytes(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dy = torch.randn_like(x)
    nc.nc_act8_layer_norm_backward(dy, F, rows, cols, cols, codes, scales, rstd, None, F, None, 0,
                                   dx, cols, dg, db, False, ws, n)
    assert bool(torch.isnan(dx[[1, 3]]).all()) and bool(torch.isfinite(dx[[0, 2, 4]]).all())
    assert bool(torch.isnan(dg).all()) and bool(torch.isfinite(db).all())


@pytest.mark.gpu
def test_gpu_no_rows_clear_or_keep_the_sums():
    cols = 100
    dg, db = torch.full((cols,), 3.0, device="cuda"), torch.full((cols,), 4.0, device="cuda")
    F = nc.DTYPE_F32
    nc.nc_layer_norm_backward(None, F, 0, cols, cols, None, cols, None, None, None, F, None, 0, None,
                              cols, dg, db, True, None, 0)
    assert bool((dg == 3).all()) and bool((db == 4).all())
    nc.nc_layer_norm_backward(None, F, 0, cols, cols, None, cols, None, None, None, F, None, 0, None,
                              cols, dg, db, False, None, 0)
    assert not bool(dg.any()) and not bool(db.any())


@pytest.mark.gpu
def test_gpu_residual_gradient_in_place_and_repeatable():
    rows, cols = 300, 3000
    bf = dict(dtype=torch.bfloat16, device="cuda")
    dy, x, dres = (torch.randn(rows, cols, **bf) for _ in range(3))
    mean, rstd = x.float().mean(1), (x.float().var(1, unbiased=False) + EPS).rsqrt()
    n = nc.nc_layer_norm_workspace_bytes(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = []
    for in_place in (False, True, False):
        dr = dres.clone()
        dx = dr if in_place else torch.empty_like(dy)
        dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        nc.nc_layer_norm_backward(dy, nc.DTYPE_BF16, rows, cols, cols, x, cols, mean, rstd, None,
                                  nc.DTYPE_BF16, dr, cols, dx, cols, dg, db, False, ws, n)
        outs.append((dx.clone(), dg, db))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
