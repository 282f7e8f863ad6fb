"""Cross entropy gradients whose logits or table gradients are long sums.

The tensor cores cut off what an accumulator cannot hold, always towards 0.  With bfloat16 a sum of 1024
products of one sign is too small by 5e-7 of its size, one of 8192 by 4e-6; twice that is allowed here.  A
product of binary16 has 22 bits instead of 16, so that of each of them something is cut off too: with u = 2^-24
the unit of a sum in [1, 2) is 2 u, and of 1024 products each loses at most that of a partial sum which is half
the final one on the average: at most 1024 u = 6e-5 of the sum.  A cut of 25 or 26 bits, which the 16 products
of an instruction are added with, makes it a quarter to a half of that; allowed is what the tests of shorter sums
allow, 4 u for each 16 products, 1.6e-5 for 1024.  Longer sums are chains of that many products, added up in binary32 (u for each),
so that nothing grows with the length.  The cases have terms of one sign, for which the cut-off adds up."""
import glob
import os
import re

import pytest
import torch

import paper_1905_10988_b200 as nc
from operator_util import CODES, TYPES, U, Placed, workspace
from test_linear_cross_entropy import Case, check_backward, check_forward


class Confident(Case):
    """Rows along their target's entry of the table: 1 - p of a target between about 1e-3 and 1e-5, logits of
    25 and more, sums of which no term is negative."""

    def __init__(self, rows, width, vocabulary, kind, out=None):
        super().__init__(rows, width, vocabulary, kind, without=0.1, scale=1.0)
        g = self.generator
        w = 1 + torch.randn(vocabulary, width, generator=g, device="cuda")
        self.w.view.copy_(w)
        w = self.w.view.double()
        size = 25 + 8 * torch.rand(rows, 1, generator=g, device="cuda")
        x = w[self.target.clamp(min=0)]
        x = size * x / x.square().sum(1, keepdim=True)
        x[self.target < 0] = float("nan")
        self.x.view.copy_(x)

    def exact(self):
        loss, lse, z, off, counts, x, w = super().exact()
        # in place of the bound for one sum of any length: that of chains of 1024
        chain = 1e-6 if self.kind == "bf16" else (1024 / 16 + 4) * 4 * U
        off = (chain + (self.width / 1024 + 2) * U) * (x.abs() @ w.abs().t())
        return loss, lse, z, off, counts, x, w


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("width", [1024, 1025, 2048, 4096, 8192, 16384])
def test_confident_rows_of_a_wide_layer(width, kind):
    c = Confident(200, width, 300, kind)
    _, lse, z, _, counts, _, _ = c.exact()
    p = torch.exp(z - lse[:, None]).gather(1, c.target.clamp(min=0)[:, None])[counts]
    assert 1e-6 < float((1 - p).min()) and float((1 - p).max()) < 1e-2
    check_forward(c)
    check_backward(c, "f32", False, False, size_of_dloss=1.0)
    check_backward(c, kind, True, True, size_of_dloss=1.0)

@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,every", [(8192, 1), (8193, 1), (50000, 2), (131072, 1), (60000, 100)])
def test_table_gradients_of_many_rows(rows, every, kind):
    # all logits 0: p = 2^-8, exact in 16 bits, and dtable is 2^-8 times the sum of the rows of x
    width, vocabulary = 72, 256
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (0.5 + torch.rand(rows, width, generator=g, device="cuda")).to(TYPES[kind])
    table = torch.zeros(vocabulary, width, dtype=TYPES[kind], device="cuda")
    target = torch.full((rows,), -1, device="cuda")
    target[::every] = 0                   # the rows that count
    lse = torch.full((rows,), float(torch.tensor(256.0, dtype=torch.float64).log()), device="cuda")
    zero, one = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    for accumulate in (False, True):
        dtable = torch.full((vocabulary, width), 3.0, device="cuda")
        size = nc.nc_linear_cross_entropy_backward_workspace_bytes(rows, width, vocabulary)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        nc.nc_linear_cross_entropy_backward(x, CODES[kind], rows, width, width, table, vocabulary, width, target, 8,
                                            1.0, lse, zero, one, None, width, dtable, nc.DTYPE_F32, width,
                                            accumulate, ws, size)
        want = x.double()[target >= 0].sum(0) / 256 + (3.0 if accumulate else 0.0)
        off = float(((dtable.double() - want).abs() / want).max())
        assert off <= 8e-6 + (rows / 8192 + 4) * U, off


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocabulary", [(87, 200, 513), (300, 1001, 2049), (1000, 520, 4000), (130, 2100, 300)])
def test_forward_of_rows_with_gaps_that_count(rows, width, vocabulary, kind):
    for without, tb in ((0.0, 8), (0.3, 4)):
        check_forward(Case(rows, width, vocabulary, kind, "gap", without=without, target_bytes=tb))


# ---- no rows -------------------------------------------------------------------------------

def test_calls_enqueue_kernels_only():
    # memory is set and copied by kernels of the library's own, but for nc_copy_* and the debug build's record
    for path in glob.glob(os.path.join(os.path.dirname(nc.LIB_PATH), "csrc", "*_kernels.cu")):
        with open(path) as f:
            found = re.findall(r"\bcudaMem(?:set|cpy)\w*", f.read())
        assert not found, (os.path.basename(path), found)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["whole", "gap", "any"])
@pytest.mark.parametrize("kind,out", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_no_rows_clear_the_table_gradient_or_leave_it(kind, out, layout):
    for vocabulary, width in ((1, 1), (700, 33), (3, 5000), (9000, 8)):
        size = nc.nc_linear_cross_entropy_backward_workspace_bytes(0, width, vocabulary)
        memory, ws = workspace(size)
        table = torch.zeros(vocabulary, width, dtype=TYPES[kind], device="cuda")
        for accumulate in (False, True):
            d = Placed((vocabulary, width), out, layout)
            nc.nc_linear_cross_entropy_backward(None, CODES[kind], 0, width, width, table, vocabulary, width, None, 8,
                                                1.0, None, None, None, table, width, d.view, CODES[out], d.ld,
                                                accumulate, ws, size)
            assert bool((d.view == (-77.0 if accumulate else 0.0)).all()) and d.untouched()


# ---- more of the shapes that sums in chains come in ------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,vocabulary,kind,out,layout", [
    (5000, 40, 700, "f16", "f16", "any"),            # dtable in chains, added to what is there
    (2500, 1100, 20000, "f16", "f32", "whole"),      # both sums in chains, several tiles for every pair
    (9000, 1300, 3000, "bf16", "bf16", "gap"),
    (20000, 100, 8000, "bf16", "f32", "any"),        # the vocabulary in two pieces
])
def test_gradients_of_sums_in_chains(rows, width, vocabulary, kind, out, layout):
    check_backward(Case(rows, width, vocabulary, kind, layout, without=0.2), out, True, True)


@pytest.mark.gpu
def test_a_layer_wider_than_the_steps_of_all_chains_in_32_bits():
    width = 1 << 24
    size = nc.nc_linear_cross_entropy_forward_workspace_bytes(1, width, 3)
    if torch.cuda.mem_get_info()[0] < size + (2 << 30):
        pytest.skip("not enough free memory")
    # whole multiples of 2^-20 of which every sum is exact; the last chain of 1024 has none, the one before many
    x = torch.ones(1, width, dtype=torch.bfloat16, device="cuda")
    x[0, -1024:] = 0
    x[0, -2048:-1024] = 8
    table = torch.empty(3, width, dtype=torch.bfloat16, device="cuda")
    for v in range(3):
        table[v] = (v + 1) * 2.0 ** -20
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    nc.nc_linear_cross_entropy_forward(x, nc.DTYPE_BF16, 1, width, width, table, 3, width,
                                       torch.zeros(1, dtype=torch.long, device="cuda"), 8, 1.0, loss, lse, ws, size)
    z = torch.tensor([(v + 1) * 2.0 ** -20 * (width - 2048 + 8 * 1024) for v in range(3)], dtype=torch.float64)
    want = float(torch.logsumexp(z, 0))
    # a chain more or less is 2^-10; exponentials and the logarithm 8 u of 48
    assert abs(float(lse) - want) <= 8 * U * 48 + 8 * U and abs(float(loss) - (want - float(z[0]))) <= 16 * U * 48
