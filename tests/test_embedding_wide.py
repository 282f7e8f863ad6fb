"""Gradients of embeddings with more than 512 tokens and rows of several slabs of columns: the sorted sums of
blocks that take one segment, of grids with several slabs, and of the joins behind them."""
import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import CODES, HALF, TINY, U, Placed, within, workspace
from test_embedding import gradient, tokens_of


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["whole", "gap", "any"])
@pytest.mark.parametrize("rows,vocabulary,cols", [(2000, 3000, 1001), (3000, 700, 2056), (1500, 9000, 4097),
                                                  (9000, 300, 520), (513, 2000, 1025), (512, 2000, 1025)])
def test_backward(rows, vocabulary, cols, layout):
    g = torch.Generator(device="cuda").manual_seed(rows)
    pairs = [("bf16", "f32"), ("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f32")]
    for i, tokens in enumerate(["mixed", "one", "few", "each", "last"]):
        kind, out = pairs[(i + cols) % len(pairs)]
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
            nc.nc_embedding_backward(t, 8, rows, y.view, CODES[kind], cols, y.ld, 0.7, vocabulary, d.view,
                                     CODES[out], d.ld, accumulate, ws, size)
            want, mag, n = gradient(t, y.view, 0.7, vocabulary)
            if accumulate:
                want = want + old
            # 0.7 in binary32 is off by U of it
            ok, by = within(d.view, want, 1.01 * ((n + 3) * U * mag + (U + HALF[out]) * want.abs()) + TINY[out])
            assert ok, (tokens, kind, out, accumulate, by)
            rest = d.view.double()[(n == 0).squeeze(1)]
            assert bool((rest == (old[(n == 0).squeeze(1)] if accumulate else 0.0)).all())
            assert d.untouched()
            assert bool((memory[:256] == 255).all()) and bool((memory[256 + size:] == 255).all())
