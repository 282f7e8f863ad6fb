"""Embedding of tokens and its gradient.

Tolerances (u = 2^-24): the forward value is one binary32 product rounded to its type; a gradient row is
a sum of n values in binary32 in some order, n u times the sum of their magnitudes, one product and one
rounding."""
import numpy as np
import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import CODES, HALF, TINY, U, Placed, address, status, within, workspace


# ---- CPU -----------------------------------------------------------------------------------

def test_the_gradients_formula_agrees_with_differences():
    rng = np.random.default_rng(1)
    table, tokens, dy = rng.standard_normal((5, 3)), np.array([4, 0, 4, -1, 2, 4]), None
    dy = rng.standard_normal((6, 3))

    def loss(table):
        rows = np.where(tokens[:, None] < 0, 0.0, 1.5 * table[np.maximum(tokens, 0)])
        return float((rows * dy).sum())

    want = np.zeros_like(table)
    for t, g in zip(tokens, dy):
        if t >= 0:
            want[t] += 1.5 * g
    h = 1e-6
    for i in range(5):
        for j in range(3):
            e = np.zeros_like(table)
            e[i, j] = h
            assert abs((loss(table + e) - loss(table - e)) / (2 * h) - want[i, j]) < 1e-7


def test_refusals_need_no_gpu():
    keep, A = address()

    def f(tokens=A, tb=8, rows=4, table=A, dt=nc.DTYPE_BF16, v=9, cols=8, ldt=8, out=A, ot=nc.DTYPE_F32,
          ldo=8):
        return nc.nc_embedding_forward(tokens, tb, rows, table, dt, v, cols, ldt, 1.0, out, ot, ldo,
                                       stream=0)

    assert status(lambda: f(dt=9)) == status(lambda: f(ot=3)) == "NC_ERR_UNSUPPORTED"
    assert status(lambda: f(tb=2)) == "NC_ERR_UNSUPPORTED"
    for kw in (dict(tokens=None), dict(table=None), dict(out=None), dict(ldt=7), dict(ldo=7), dict(v=0)):
        assert status(lambda: f(**kw)) == "NC_ERR_INVALID", kw
    for kw in (dict(tokens=A + 4), dict(table=A + 1), dict(out=A + 2), dict(tokens=A + 2, tb=4)):
        assert status(lambda: f(**kw)) == "NC_ERR_ALIGN", kw
    for kw in (dict(rows=1 << 31), dict(v=1 << 31), dict(cols=1 << 31, ldt=1 << 31, ldo=1 << 31)):
        assert status(lambda: f(**kw)) == "NC_ERR_TOO_LARGE", kw
    assert status(lambda: f(rows=0)) == status(lambda: f(cols=0)) == "NC_OK"

    def b(tokens=A, tb=8, rows=4, dy=A, dt=nc.DTYPE_BF16, cols=8, lddy=8, v=9, out=A, ot=nc.DTYPE_F32,
          ldo=8, ws=A, size=1 << 20):
        return nc.nc_embedding_backward(tokens, tb, rows, dy, dt, cols, lddy, 1.0, v, out, ot, ldo, False,
                                        ws, size, stream=0)

    assert status(lambda: b(dt=9)) == status(lambda: b(ot=3)) == status(lambda: b(tb=1)) == "NC_ERR_UNSUPPORTED"
    for kw in (dict(tokens=None), dict(dy=None), dict(out=None), dict(lddy=7), dict(ldo=7), dict(ws=None)):
        assert status(lambda: b(**kw)) == "NC_ERR_INVALID", kw
    for kw in (dict(tokens=A + 4), dict(dy=A + 1), dict(out=A + 2), dict(ws=A + 8)):
        assert status(lambda: b(**kw)) == "NC_ERR_ALIGN", kw
    for kw in (dict(rows=1 << 31), dict(v=1 << 31), dict(cols=1 << 24, lddy=1 << 24, ldo=1 << 24)):
        assert status(lambda: b(**kw)) == "NC_ERR_TOO_LARGE", kw
    assert status(lambda: b(size=nc.nc_embedding_backward_workspace_bytes(4, 9, 8) - 1)) == "NC_ERR_WORKSPACE"
    assert status(lambda: b(cols=0)) == status(lambda: b(v=0)) == "NC_OK"
    assert nc.nc_embedding_backward_workspace_bytes(1 << 31, 9, 8) == 0


# ---- GPU -----------------------------------------------------------------------------------

def tokens_of(kind, rows, vocabulary, g):
    dev = dict(device="cuda")
    if kind == "one":
        return torch.full((rows,), vocabulary // 2, **dev)
    if kind == "last":
        return torch.full((rows,), vocabulary - 1, **dev)
    if kind == "none":
        return -1 - torch.randint(0, 9, (rows,), generator=g, **dev)
    if kind == "each":
        return torch.arange(rows, **dev).flip(0) % vocabulary
    t = torch.randint(0, 3 if kind == "few" else vocabulary, (rows,), generator=g, **dev) % vocabulary
    if kind == "mixed":
        t[torch.rand(rows, generator=g, **dev) < 0.2] = -1
        t[torch.rand(rows, generator=g, **dev) < 0.1] = vocabulary
        t[::7] = min(3, vocabulary - 1)
    return t


def gradient(tokens, dy, scale, vocabulary):
    """-> sums, sums of magnitudes, tokens of a row; in 64 bits"""
    there = (tokens >= 0) & (tokens < vocabulary)
    at, d = tokens[there], dy[there].double()
    want = torch.zeros(vocabulary, dy.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    want.index_add_(0, at, scale * d)
    size.index_add_(0, at, abs(scale) * d.abs())
    return want, size, torch.bincount(at, minlength=vocabulary).double().unsqueeze(1)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["whole", "gap", "any"])
@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "f32"),
                                      ("bf16", "bf16"), ("bf16", "f16"), ("f16", "f32"), ("f16", "bf16"),
                                      ("f16", "f16")])
def test_forward(kind, out, layout):
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows, vocabulary, cols, token_bytes in [(1, 1, 1, 8), (5, 9, 7, 4), (33, 40, 8, 8), (70, 300, 1001, 4),
                                                (3, 50, 1024, 8), (9, 20, 4097, 8), (400, 11, 264, 4)]:
        table = Placed((vocabulary, cols), kind, layout,
                       torch.randn(vocabulary, cols, generator=g, device="cuda"))
        t = tokens_of("mixed", rows, vocabulary, g)
        o = Placed((rows, cols), out, layout)
        nc.nc_embedding_forward(t if token_bytes == 8 else t.int(), token_bytes, rows, table.view,
                                CODES[kind], vocabulary, cols, table.ld, 0.3, o.view, CODES[out], o.ld)
        in_it = ((t >= 0) & (t < vocabulary)).unsqueeze(1)
        want = float(np.float32(0.3)) * table.view.double()[t.clamp(0, vocabulary - 1)]
        ok, by = within(torch.where(in_it, o.view.double(), want), want,
                        (U + HALF[out]) * 1.01 * want.abs() + TINY[out])
        assert ok, (rows, vocabulary, cols, by)
        assert bool((o.view[t < 0] == 0).all()) and bool(o.view[t >= vocabulary].isnan().all())
        assert o.untouched()


SIZES = [(1, 1, 1), (31, 9, 8), (33, 1000, 33), (300, 40, 1001), (257, 5000, 1024), (8192, 700, 24),
         (8193, 20000, 9), (40000, 300, 40), (70001, 100003, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["whole", "gap", "any"])
@pytest.mark.parametrize("rows,vocabulary,cols", SIZES)
def test_backward(rows, vocabulary, cols, layout):
    g = torch.Generator(device="cuda").manual_seed(2)
    pairs = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16"),
             ("f32", "bf16"), ("f32", "f16"), ("bf16", "f16"), ("f16", "bf16")]
    for i, tokens in enumerate(["mixed", "one", "few", "each", "none", "last"]):
        kind, out = pairs[(i + rows) % len(pairs)]
        t = tokens_of(tokens, rows, vocabulary, g)
        dy = torch.randn(rows, cols, generator=g, device="cuda")
        dy[(t < 0) | (t >= vocabulary)] = float("nan")
        y = Placed((rows, cols), kind, layout, dy)
        for accumulate in (False, True):
            d = Placed((vocabulary, cols), out, layout)
            if accumulate:
                d.view.copy_(torch.randn(vocabulary, cols, generator=g, device="cuda"))
            old = d.view.double()
            size = nc.nc_embedding_backward_workspace_bytes(rows, vocabulary, cols)
            memory, ws = workspace(size)
            nc.nc_embedding_backward(t if i % 2 else t.int(), 8 if i % 2 else 4, rows, y.view, CODES[kind],
                                     cols, y.ld, -1.25, vocabulary, d.view, CODES[out], d.ld, accumulate,
                                     ws, size)
            want, mag, n = gradient(t, y.view, -1.25, vocabulary)
            if accumulate:
                want = want + old
            ok, by = within(d.view, want, 1.01 * ((n + 2) * U * mag + (U + HALF[out]) * want.abs()) + TINY[out])
            assert ok, (tokens, kind, out, accumulate, by)
            if accumulate:
                assert bool((d.view.double() == old)[(n == 0).squeeze(1)].all())
            else:
                assert bool((d.view[(n == 0).squeeze(1)] == 0).all())
            assert d.untouched()
            assert bool((memory[:256] == 255).all()) and bool((memory[256 + size:] == 255).all())


@pytest.mark.gpu
def test_no_rows_clear_the_gradient_or_leave_it():
    size = nc.nc_embedding_backward_workspace_bytes(0, 37, 11)
    memory, ws = workspace(size)
    for accumulate in (False, True):
        d = Placed((37, 11), "f32", "any")
        nc.nc_embedding_backward(None, 8, 0, None, nc.DTYPE_BF16, 11, 11, 1.0, 37, d.view, nc.DTYPE_F32,
                                 d.ld, accumulate, ws, size)
        assert bool((d.view == (-77.0 if accumulate else 0.0)).all()) and d.untouched()


@pytest.mark.gpu
def test_gradient_is_the_same_bits_and_captured_and_on_two_streams():
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, vocabulary, cols = 9000, 500, 520
    t = tokens_of("mixed", rows, vocabulary, g)
    dy = torch.randn(rows, cols, generator=g, device="cuda")
    size = nc.nc_embedding_backward_workspace_bytes(rows, vocabulary, cols)
    table = torch.randn(vocabulary, cols, generator=g, device="cuda")

    def call(out, rows_out, ws):
        nc.nc_embedding_backward(t, 8, rows, dy, nc.DTYPE_F32, cols, cols, 1.0, vocabulary, out,
                                 nc.DTYPE_F32, cols, False, ws, size)
        nc.nc_embedding_forward(t, 8, rows, table, nc.DTYPE_F32, vocabulary, cols, cols, 2.0, rows_out,
                                nc.DTYPE_F32, cols)

    outs = [(torch.empty(vocabulary, cols, device="cuda"), torch.empty(rows, cols, device="cuda"),
             torch.empty(size, dtype=torch.uint8, device="cuda")) for _ in range(4)]
    call(*outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, o in zip(streams, outs[1:3]):
            with torch.cuda.stream(s):
                call(*o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*outs[3])
    outs[3][0].fill_(9)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o[0], outs[0][0])
        assert torch.equal(o[1].nan_to_num(5.0), outs[0][1].nan_to_num(5.0))
    # the captured call reads its inputs when it is replayed
    t.copy_(t.flip(0))
    dy.mul_(2)
    graph.replay()
    call(*outs[0])
    torch.cuda.synchronize()
    assert torch.equal(outs[3][0], outs[0][0])


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    vocabulary, cols = 600_000, 4096
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("not enough free memory")
    t = torch.tensor([vocabulary - 1, 5, 530_000, vocabulary - 1, 524_288], device="cuda")
    table = torch.zeros(vocabulary, cols, dtype=torch.bfloat16, device="cuda")
    table[t] = torch.randn(5, cols, device="cuda").bfloat16()
    out = torch.empty(5, cols, dtype=torch.bfloat16, device="cuda")
    nc.nc_embedding_forward(t, 8, 5, table, nc.DTYPE_BF16, vocabulary, cols, cols, 1.0, out, nc.DTYPE_BF16, cols)
    assert torch.equal(out, table[t])
    size = nc.nc_embedding_backward_workspace_bytes(5, vocabulary, cols)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want = torch.zeros(5, cols, device="cuda")
    want += out.float()
    want[0] *= 2
    want[3] = want[0]
    table.fill_(3.0)
    nc.nc_embedding_backward(t, 8, 5, out, nc.DTYPE_BF16, cols, cols, 1.0, vocabulary, table, nc.DTYPE_BF16,
                             cols, False, ws, size)
    assert torch.equal(table[t].float(), want.bfloat16().float())
    table[t] = 0
    assert int(table.view(torch.int16).count_nonzero()) == 0
