"""Softmax cross entropy of a linear output layer, and its gradient.

Tolerances (u = 2^-24): a logit is a sum of width products which the tensor cores add 16 at a time to a
binary32 sum that is cut off instead of rounded: off by at most (width / 16 + 4) * 4 u times the sum of
the terms' magnitudes.  The exponentials take their argument with four roundings (8 u times the sizes
in it) and are right to 4 u; sums of v of them in binary32 to v u.  dz is rounded to 16 bits once, and
every sum over it is one of the tensor cores again; the results are rounded once."""
import numpy as np
import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import CODES, HALF, TINY, TYPES, U, Placed, address, status, within, workspace


# ---- CPU -----------------------------------------------------------------------------------

def plain(x, w, target, scale):
    """-> loss, lse, logits, which rows count; in the inputs' precision"""
    z = scale * x @ w.t()
    counts = target >= 0
    lse = torch.logsumexp(z, 1)
    hit = z.gather(1, target.clamp(0, w.shape[0] - 1).unsqueeze(1)).squeeze(1)
    zero = torch.zeros_like(lse)
    return torch.where(counts, lse - hit, zero), torch.where(counts, lse, zero), z, counts


def test_the_gradients_formula_agrees_with_differences():
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(4, 3, generator=g).double(), torch.randn(5, 3, generator=g).double()
    target = torch.tensor([4, -1, 0, 2])
    dl, ds = torch.randn(4, generator=g).double(), torch.randn(4, generator=g).double()

    def total(x, w):
        loss, lse, _, _ = plain(x, w, target, 0.7)
        return float((dl * loss + ds * lse).sum())

    _, lse, z, counts = plain(x, w, target, 0.7)
    dz = torch.exp(z - lse[:, None]) * (dl + ds)[:, None]
    dz[torch.arange(4), target.clamp(min=0)] -= dl
    dz *= counts[:, None]
    dx, dw, h = 0.7 * dz @ w, 0.7 * dz.t() @ x, 1e-6
    for m, d, swap in ((x, dx, 0), (w, dw, 1)):
        for i in range(m.shape[0]):
            for j in range(m.shape[1]):
                e = torch.zeros_like(m)
                e[i, j] = h
                up, down = (total(x + e, w), total(x - e, w)) if not swap else (total(x, w + e), total(x, w - e))
                assert abs((up - down) / (2 * h) - d[i, j]) < 1e-6


def test_refusals_need_no_gpu():
    keep, A = address()
    good = dict(x=A, dtype=nc.DTYPE_BF16, rows=4, width=16, ldx=16, table=A, v=8, ldt=16, targets=A, tb=8,
                scale=1.0)

    def f(loss=A, lse=A, ws=A, size=1 << 20, **kw):
        k = dict(good, **kw)
        return nc.nc_linear_cross_entropy_forward(k["x"], k["dtype"], k["rows"], k["width"], k["ldx"],
                                                  k["table"], k["v"], k["ldt"], k["targets"], k["tb"],
                                                  k["scale"], loss, lse, ws, size, stream=0)

    def b(lse=A, dloss=A, dlse=None, dx=A, lddx=16, dt=A, dtt=nc.DTYPE_F32, lddt=16, ws=A, size=1 << 20, **kw):
        k = dict(good, **kw)
        return nc.nc_linear_cross_entropy_backward(k["x"], k["dtype"], k["rows"], k["width"], k["ldx"],
                                                   k["table"], k["v"], k["ldt"], k["targets"], k["tb"],
                                                   k["scale"], lse, dloss, dlse, dx, lddx, dt, dtt, lddt,
                                                   False, ws, size, stream=0)

    for call in (f, b):
        for kw in (dict(dtype=nc.DTYPE_F32), dict(dtype=7), dict(tb=2)):
            assert status(lambda: call(**kw)) == "NC_ERR_UNSUPPORTED", kw
        for kw in (dict(x=None), dict(table=None), dict(targets=None), dict(ldx=15), dict(ldt=15), dict(ws=None),
                   dict(width=0), dict(v=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                   dict(scale=float("inf")), dict(scale=2.5e38)):
            assert status(lambda: call(**kw)) == "NC_ERR_INVALID", kw
        for kw in (dict(x=A + 1), dict(table=A + 1), dict(targets=A + 4), dict(ws=A + 16), dict(lse=A + 2)):
            assert status(lambda: call(**kw)) == "NC_ERR_ALIGN", kw
        for kw in (dict(rows=1 << 31), dict(v=1 << 31), dict(width=1 << 31, ldx=1 << 31, ldt=1 << 31)):
            assert status(lambda: call(**kw)) == "NC_ERR_TOO_LARGE", kw
        assert status(lambda: call(size=100)) == "NC_ERR_WORKSPACE"
    assert status(lambda: f(loss=None)) == status(lambda: f(lse=None)) == "NC_ERR_INVALID"
    assert status(lambda: f(rows=0)) == "NC_OK"
    assert status(lambda: b(dtt=nc.DTYPE_F16)) == "NC_ERR_UNSUPPORTED"
    for kw in (dict(lddx=15), dict(lddt=15), dict(lse=None), dict(dloss=None)):
        assert status(lambda: b(**kw)) == "NC_ERR_INVALID", kw
    for kw in (dict(dx=A + 1), dict(dt=A + 2), dict(dloss=A + 1), dict(dlse=A + 2)):
        assert status(lambda: b(**kw)) == "NC_ERR_ALIGN", kw
    assert status(lambda: b(dx=None, dt=None)) == "NC_OK"
    for h in (nc.nc_linear_cross_entropy_forward_workspace_bytes,
              nc.nc_linear_cross_entropy_backward_workspace_bytes):
        assert h(1 << 31, 8, 8) == 0 and h(1, 1, 1) > 0


def test_backward_workspace_does_not_grow_with_the_vocabulary():
    # rows * vocabulary would be 4 GB in 16 bits
    h = nc.nc_linear_cross_entropy_backward_workspace_bytes
    assert h(16384, 1024, 131072) == h(16384, 1024, 65536) < 1 << 29


# ---- GPU -----------------------------------------------------------------------------------

class Case:
    def __init__(self, rows, width, vocabulary, kind, layout="whole", spread=2.0, without=0.3, seed=1,
                 target_bytes=8, scale=0.8):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*s):
            return torch.randn(*s, generator=g, device="cuda")

        self.rows, self.width, self.vocabulary, self.kind = rows, width, vocabulary, kind
        self.scale, self.generator, self.layout = float(np.float32(scale)), g, layout
        self.target = torch.randint(0, vocabulary, (rows,), generator=g, device="cuda")
        w = spread / width ** 0.5 * normal(vocabulary, width)
        x = normal(rows, width) + torch.rand(rows, 1, generator=g, device="cuda") * w[self.target]
        self.target[torch.rand(rows, generator=g, device="cuda") < without] = -3
        x[self.target < 0] = float("nan")
        self.x, self.w = Placed((rows, width), kind, layout, x), Placed((vocabulary, width), kind, layout, w)
        self.given = self.target if target_bytes == 8 else self.target.int()
        self.tb = target_bytes

    def forward(self):
        c = self
        loss, lse = (torch.full((c.rows + 2,), 7.0, device="cuda") for _ in range(2))
        size = nc.nc_linear_cross_entropy_forward_workspace_bytes(c.rows, c.width, c.vocabulary)
        memory, ws = workspace(size)
        nc.nc_linear_cross_entropy_forward(c.x.view, CODES[c.kind], c.rows, c.width, c.x.ld, c.w.view,
                                           c.vocabulary, c.w.ld, c.given, c.tb, c.scale, loss[1:], lse[1:],
                                           ws, size)
        torch.cuda.synchronize()
        assert bool((memory[:256] == 255).all()) and bool((memory[256 + size:] == 255).all())
        assert float(loss[0]) == float(loss[-1]) == float(lse[0]) == float(lse[-1]) == 7.0
        return loss[1:-1], lse[1:-1]

    def exact(self):
        """loss, lse, logits in 64 bits, and what a logit may be off by"""
        x = torch.where(self.target[:, None] >= 0, self.x.view.double(), 0.0)
        w = self.w.view.double()
        loss, lse, z, counts = plain(x, w, self.target, self.scale)
        off = (self.width / 16 + 4) * 4 * U * self.scale * (x.abs() @ w.abs().t())
        return loss, lse, z, off, counts, x, w


def check_forward(c):
    loss, lse = c.forward()
    want, want_lse, z, off, counts, _, _ = c.exact()
    tol = off.amax(1) + (c.vocabulary + 16) * U + 8 * U * (want_lse.abs() + z.abs().amax(1)) + 1e-30
    ok, by = within(lse, want_lse, tol)
    assert ok, ("lse", by)
    ok, by = within(loss, want, 2 * tol)
    assert ok, ("loss", by)
    assert bool((loss[~counts] == 0).all()) and bool((lse[~counts] == 0).all())


def check_backward(c, out, accumulate, with_dlse, want_dx=True, want_dtable=True, size_of_dloss=1e-3):
    _, lse, z, off, counts, x, w = c.exact()
    g = c.generator
    dl = size_of_dloss * (0.5 + torch.rand(c.rows, generator=g, device="cuda"))
    ds = size_of_dloss * torch.randn(c.rows, generator=g, device="cuda")
    dl[~counts] = ds[~counts] = float("nan")
    lse32 = torch.where(counts, lse, float("nan")).float()
    dx = Placed((c.rows, c.width), c.kind, c.layout)
    dt = Placed((c.vocabulary, c.width), out, c.layout)
    if accumulate:
        dt.view.copy_(size_of_dloss * torch.randn(c.vocabulary, c.width, generator=g, device="cuda"))
    old = dt.view.double()
    size = nc.nc_linear_cross_entropy_backward_workspace_bytes(c.rows, c.width, c.vocabulary)
    memory, ws = workspace(size)
    nc.nc_linear_cross_entropy_backward(
        c.x.view, CODES[c.kind], c.rows, c.width, c.x.ld, c.w.view, c.vocabulary, c.w.ld, c.given, c.tb,
        c.scale, lse32, dl, ds if with_dlse else None, dx.view if want_dx else None, dx.ld,
        dt.view if want_dtable else None, CODES[out], dt.ld, accumulate, ws, size)
    torch.cuda.synchronize()
    assert bool((memory[:256] == 255).all()) and bool((memory[256 + size:] == 255).all())
    a = torch.where(counts, dl.double(), 0.0)[:, None]
    b = a + (torch.where(counts, ds.double(), 0.0)[:, None] if with_dlse else 0.0)
    p = torch.exp(z - lse32.double().nan_to_num(0.0)[:, None]) * counts[:, None]
    hot = torch.zeros_like(p)
    hot[torch.arange(c.rows, device="cuda"), c.target.clamp(min=0)] = 1.0
    hot *= counts[:, None]
    dz = p * b - hot * a
    largest = float(torch.maximum(torch.maximum(a.abs(), b.abs()), (b - a).abs()).max()) if c.rows else 0.0
    edz = HALF[c.kind] * dz.abs() + largest * (2.0 ** -38 if c.kind == "f16" else 2.0 ** -120) * counts[:, None]
    edz += (p * b.abs() + hot * a.abs()) * (off + 8 * U * (2 + z.abs() + lse.abs()[:, None]))
    if want_dx:
        want = c.scale * dz @ w
        tol = c.scale * (edz @ w.abs() + (c.vocabulary / 16 + 80) * 4 * U * (dz.abs() @ w.abs()))
        ok, by = within(dx.view, want, 1.01 * (tol + HALF[c.kind] * want.abs()) + TINY[c.kind])
        assert ok, ("dx", by)
        assert bool((dx.view[~counts] == 0).all()) and dx.untouched()
    else:
        assert bool((dx.view == -77.0).all())
    if want_dtable:
        want = c.scale * dz.t() @ x + (old if accumulate else 0.0)
        tol = c.scale * (edz.t() @ x.abs() + (c.rows / 16 + 8) * 4 * U * (dz.abs().t() @ x.abs()))
        ok, by = within(dt.view, want, 1.01 * (tol + (HALF[out] + 2 * U) * want.abs()) + TINY[out])
        assert ok, ("dtable", by)
        assert dt.untouched()
    else:
        assert bool((dt.view == -77.0).all())


SIZES = [(1, 1, 1), (1, 64, 1000), (3, 7, 5), (64, 128, 256), (87, 200, 513), (256, 72, 255), (300, 1001, 2049),
         (1000, 520, 4000), (2, 4096, 33), (513, 64, 40000)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocabulary", SIZES)
def test_forward(rows, width, vocabulary, kind):
    for layout, without, tb in (("whole", 0.0, 8), ("any", 0.5, 4), ("gap", 1.0, 8)):
        check_forward(Case(rows, width, vocabulary, kind, layout, without=without, target_bytes=tb))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocabulary", SIZES)
def test_backward(rows, width, vocabulary, kind):
    check_backward(Case(rows, width, vocabulary, kind), kind, False, False)
    check_backward(Case(rows, width, vocabulary, kind, "any", target_bytes=4), "f32", True, True)
    check_backward(Case(rows, width, vocabulary, kind, "gap", without=0.0), kind, True, True)
    check_backward(Case(rows, width, vocabulary, kind, without=1.0), "f32", False, True)


@pytest.mark.gpu
def test_one_of_the_gradients_alone():
    for out in ("f16", "f32"):
        check_backward(Case(300, 200, 700, "f16"), out, False, False, want_dx=False)
        check_backward(Case(300, 200, 700, "f16"), out, False, False, want_dtable=False)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["whole", "any"])
def test_pieces_of_the_vocabulary(layout):
    # rows enough that dz is worked through in three pieces, the last one ragged
    check_forward(Case(66000, 40, 4500, "bf16", layout))
    check_backward(Case(66000, 40, 4500, "bf16", layout), "bf16", False, True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1e-30, 1e-8, 1e4, 1e30])
def test_any_size_of_the_incoming_gradient(kind, size):
    if kind == "f16" and size != 1e-8:
        return                            # the result itself leaves binary16
    check_backward(Case(200, 96, 300, kind, without=0.1), "f32", False, True, size_of_dloss=size)


@pytest.mark.gpu
def test_large_logits_and_confident_rows():
    check_forward(Case(200, 128, 1000, "bf16", spread=60.0))
    check_backward(Case(200, 128, 1000, "bf16", spread=60.0), "bf16", False, False)


@pytest.mark.gpu
def test_targets_beyond_the_vocabulary_are_nan_and_no_gradient_of_zero_is():
    c = Case(40, 64, 300, "bf16", without=0.0)
    c.target[7] = 300
    c.target[9] = 1 << 40
    loss, lse = c.forward()
    assert loss.isnan().nonzero().flatten().tolist() == [7, 9] and not bool(lse.isnan().any())
    size = nc.nc_linear_cross_entropy_backward_workspace_bytes(40, 64, 300)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    dx, dt = torch.empty(40, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(300, 64, device="cuda")

    def call(dloss):
        nc.nc_linear_cross_entropy_backward(c.x.view, nc.DTYPE_BF16, 40, 64, c.x.ld, c.w.view, 300, c.w.ld,
                                            c.target, 8, 1.0, lse, dloss, None, dx, 64, dt, nc.DTYPE_F32,
                                            64, False, ws, size)

    call(torch.ones(40, device="cuda"))
    assert dx.isnan().all(1).nonzero().flatten().tolist() == [7, 9] and bool(dt.isnan().all())
    c.target.clamp_(max=299)
    call(torch.zeros(40, device="cuda"))
    assert bool((dx == 0).all()) and bool((dt == 0).all())
    # a gradient that is not finite stays with its row of dx
    dloss = torch.ones(40, device="cuda")
    dloss[3] = float("inf")
    call(dloss)
    bad = (~dx.isfinite()).any(1).nonzero().flatten().tolist()
    assert bad == [3]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_gradient_that_is_not_finite_leaves_the_other_rows_alone(kind, bad):
    c = Case(40, 64, 300, kind, without=0.0)
    _, lse = c.forward()
    size = nc.nc_linear_cross_entropy_backward_workspace_bytes(40, 64, 300)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    dloss, got = torch.full((40,), 20.0, device="cuda"), []
    for i in range(2):
        dx = torch.empty(40, 64, dtype=TYPES[kind], device="cuda")
        nc.nc_linear_cross_entropy_backward(c.x.view, CODES[kind], 40, 64, c.x.ld, c.w.view, 300, c.w.ld,
                                            c.target, 8, c.scale, lse, dloss, None, dx, 64, None, CODES[kind],
                                            64, False, ws, size)
        got.append(dx)
        dloss[3] = bad
    keep = torch.arange(40, device="cuda") != 3
    assert bool(got[0].isfinite().all()) and torch.equal(got[0][keep], got[1][keep])
    assert not bool(got[1][3].isfinite().any())


@pytest.mark.gpu
def test_infinities_reach_their_own_rows_only():
    c = Case(50, 64, 300, "f16", without=0.0)
    c.x.view[4, 5] = float("inf")
    c.x.view[6] = float("nan")
    loss, lse = c.forward()
    assert (~loss.isfinite()).nonzero().flatten().tolist() == [4, 6]
    # a vocabulary entry that no row can take: its logits are -inf
    c = Case(50, 64, 300, "bf16", without=0.0)
    c.x.view.copy_(c.x.view.abs() + 0.1)
    c.w.view[17] = float("-inf")
    c.target[c.target == 17] = 0
    loss, lse = c.forward()
    w = c.w.view.double()
    keep = torch.arange(300, device="cuda") != 17
    want = torch.logsumexp(c.scale * c.x.view.double() @ w[keep].t(), 1)
    assert bool(loss.isfinite().all()) and float((lse - want).abs().max()) < 1e-3


@pytest.mark.gpu
def test_the_same_bits_captured_and_on_two_streams():
    c = Case(700, 200, 3000, "bf16", without=0.2)
    _, lse = c.forward()
    d = torch.rand(700, device="cuda")
    size = nc.nc_linear_cross_entropy_backward_workspace_bytes(700, 200, 3000)
    fsize = nc.nc_linear_cross_entropy_forward_workspace_bytes(700, 200, 3000)
    like = dict(dtype=torch.bfloat16, device="cuda")

    def buffers():
        return (torch.empty(700, 200, **like), torch.empty(3000, 200, **like),
                torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(700, device="cuda"),
                torch.empty(700, device="cuda"), torch.empty(fsize, dtype=torch.uint8, device="cuda"))

    def call(dx, dt, ws, loss, out_lse, fws):
        nc.nc_linear_cross_entropy_forward(c.x.view, nc.DTYPE_BF16, 700, 200, c.x.ld, c.w.view, 3000, c.w.ld,
                                           c.target, 8, c.scale, loss, out_lse, fws, fsize)
        nc.nc_linear_cross_entropy_backward(c.x.view, nc.DTYPE_BF16, 700, 200, c.x.ld, c.w.view, 3000, c.w.ld,
                                            c.target, 8, c.scale, out_lse, d, None, dx, 200, dt,
                                            nc.DTYPE_BF16, 200, False, ws, size)

    sets = [buffers() for _ in range(4)]
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
        for i in (0, 1, 3, 4):
            assert torch.equal(b[i], sets[0][i]), i
    c.target.copy_(c.target.flip(0))              # read when the graph is replayed
    c.x.view.copy_(c.x.view.flip(0))
    graph.replay()
    call(*sets[0])
    torch.cuda.synchronize()
    assert torch.equal(sets[3][1], sets[0][1]) and torch.equal(sets[3][3], sets[0][3])


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    # the table has more than 2^31 values; every row's weight is on two entries far apart
    vocabulary, width, rows = 530_000, 4096, 64
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("not enough free memory")
    w = torch.zeros(vocabulary, width, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    i = torch.arange(rows, device="cuda")
    target = vocabulary - 1 - 3 * i
    x[i, i] = 8.0
    w[target, i] = 8.0
    w[i, i] = 8.0
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    size = nc.nc_linear_cross_entropy_forward_workspace_bytes(rows, width, vocabulary)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    nc.nc_linear_cross_entropy_forward(x, nc.DTYPE_BF16, rows, width, width, w, vocabulary, width, target, 8,
                                       1.0, loss, lse, ws, size)
    # two logits of 64, all others 0
    want = 64 + np.log(2 + (vocabulary - 2) * np.exp(-64.0))
    assert float((lse - want).abs().max()) < 1e-4 and float((loss - (want - 64)).abs().max()) < 1e-4
    size = nc.nc_linear_cross_entropy_backward_workspace_bytes(rows, width, vocabulary)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    dt = torch.full((vocabulary, width), 9.0, dtype=torch.bfloat16, device="cuda")
    dx = torch.empty_like(x)
    nc.nc_linear_cross_entropy_backward(x, nc.DTYPE_BF16, rows, width, width, w, vocabulary, width, target, 8,
                                        1.0, lse, torch.ones(rows, device="cuda"), None, dx, width, dt,
                                        nc.DTYPE_BF16, width, False, ws, size)
    # dz is -1/2 at the target and 1/2 at the other entry
    assert float((dt[target, i].float() + 4).abs().max()) < 0.02
    assert float((dt[i, i].float() - 4).abs().max()) < 0.02
    assert float(dx.float().abs().max()) < 0.05
    dt[target, i] = 0
    dt[i, i] = 0
    assert float(dt.abs().max()) < 1e-20
