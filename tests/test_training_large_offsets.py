"""The training operators where element offsets pass 32 bits: rows far into a large matrix are compared
with calls on those rows alone."""
import pytest
import torch

import paper_1905_10988_b200 as nc

pytestmark = pytest.mark.gpu
B, F = nc.DTYPE_BF16, nc.DTYPE_F32


def u8(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def matrix(rows, cols, seed):
    """random bfloat16 rows, the last 700 of their own"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = torch.randn(4096, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 4096):
        x[i:i + 4096] = block[:min(4096, rows - i)]
    x[-700:] = torch.randn(700, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    return x


@pytest.mark.parametrize("rows,cols", [(70001, 32768), (70001, 32801)])
def test_checkpoint_far_into_a_matrix(rows, cols):
    assert rows * cols > 1 << 31
    x = matrix(rows, cols, 1)
    codes, scales = u8(nc.nc_act8_code_bytes(rows, cols)), u8(nc.nc_act8_scale_bytes(rows, cols))
    nc.nc_act8_compress(x, B, rows, cols, cols, nc.ROUND_NEAREST, 0, 0, codes, scales)
    n, pitch = 5, -(-cols // 32) * 32
    tail = x[-n:].clone()
    tcodes, tscales = u8(nc.nc_act8_code_bytes(n, cols)), u8(nc.nc_act8_scale_bytes(n, cols))
    nc.nc_act8_compress(tail, B, n, cols, cols, nc.ROUND_NEAREST, 0, 0, tcodes, tscales)
    assert torch.equal(codes.view(rows, pitch)[-n:].reshape(-1), tcodes)
    assert torch.equal(scales[:rows * pitch // 32].view(rows, -1)[-n:].reshape(-1),
                       tscales[:n * pitch // 32])
    back, tback = torch.zeros_like(x), torch.empty_like(tail)
    nc.nc_act8_decompress(codes, scales, rows, cols, back, B, cols)
    nc.nc_act8_decompress(tcodes, tscales, n, cols, tback, B, cols)
    assert torch.equal(back[-n:], tback) and torch.equal(back[4096:8192], back[:4096])


@pytest.mark.parametrize("rows,cols", [(280001, 8192), (270001, 8001)])
def test_norm_far_into_a_matrix(rows, cols):
    assert rows * cols > 1 << 31
    x, dy = matrix(rows, cols, 2), matrix(rows, cols, 3)
    f32 = dict(dtype=torch.float32, device="cuda")

    def forward_and_backward(x, dy):
        r = x.shape[0]
        y, mean, rstd = torch.empty_like(x), torch.empty(r, **f32), torch.empty(r, **f32)
        codes, scales = u8(nc.nc_act8_code_bytes(r, cols)), u8(nc.nc_act8_scale_bytes(r, cols))
        nc.nc_layer_norm_forward(x, B, r, cols, cols, None, None, F, 1e-5, y, cols, mean, rstd, codes,
                                 scales, nc.ROUND_NEAREST, 0, 0)
        dx, dg, db = torch.empty_like(x), torch.empty(cols, **f32), torch.empty(cols, **f32)
        size = nc.nc_layer_norm_workspace_bytes(r, cols)
        nc.nc_act8_layer_norm_backward(dy, B, r, cols, cols, codes, scales, rstd, None, F, dy, cols, dx,
                                       cols, dg, db, False, u8(size), size)
        return y, dx, mean, rstd

    whole = [v[-600:].clone() for v in forward_and_backward(x, dy)]
    tail = forward_and_backward(x[-600:].clone(), dy[-600:].clone())     # the same kernels
    assert all(torch.equal(p, q) for p, q in zip(whole, tail))


@pytest.mark.parametrize("n", [8192, 8193])
def test_weight_gradient_far_into_a_matrix(n):
    t, k = 270001, 40
    assert t * n > 1 << 31
    dy = matrix(t, n, 4)
    x = torch.randn(t, k, device="cuda")
    codes, scales = u8(nc.nc_act8_code_bytes(t, k)), u8(nc.nc_act8_scale_bytes(t, k))
    nc.nc_act8_compress(x, F, t, k, k, nc.ROUND_NEAREST, 0, 0, codes, scales)
    nc.nc_act8_decompress(codes, scales, t, k, x, F, k)
    size = nc.nc_act8_weight_grad_workspace_bytes(t, n, k)
    dw, db = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    nc.nc_act8_weight_grad(dy, t, n, n, codes, scales, k, None, None, F, dw, F, k, db, False, u8(size),
                           size)
    for cols in (slice(0, 16), slice(n - 16, n)):
        d = dy[:, cols].double()
        # chains of 8192 tokens, parts added in binary32: within 2^-23 * 2/3 * 512 of the norm
        want = d.t() @ x.double()
        assert float((dw[cols].double() - want).norm() / want.norm()) < 4.1e-5
        # 37 ranges or more, eight chains of additions in each, and sums of those
        sums = d.sum(0)
        assert bool(((db[cols].double() - sums).abs() <= (t / 37 / 8 + 60) * 2.0 ** -24 * d.abs().sum(0)).all())
