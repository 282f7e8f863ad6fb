"""The training step around the 8-bit checkpoints: its gradients against a 64-bit step, graph capture
of the operators, and a short training run with compressed gradients."""
import numpy as np
import pytest
import torch

import act8_reference as ref

pytestmark = pytest.mark.gpu


def _plain_step(block, x, dy):
    """Gradients of the same block in float64 with nothing kept in 8 bits."""
    p = {n: getattr(block, n).double().requires_grad_() for n in block.NAMES}
    x = x.double().requires_grad_()
    mean = x.mean(1, keepdim=True)
    xh = (x - mean) / ((x - mean).square().mean(1, keepdim=True) + 1e-5).sqrt()
    h = (xh * p["gamma"] + p["beta"]) @ p["w1"].t() + p["b1"]
    u = 0.5 * h * (1 + torch.erf(h / 2 ** 0.5))
    y = x + u @ p["w2"].t() + p["b2"]
    (y * dy.double()).sum().backward()
    return y.detach(), x.grad, {n: v.grad for n, v in p.items()}


@pytest.mark.parametrize("tokens,width,hidden", [(300, 96, 200), (1024, 256, 1024)])
def test_gradients_are_near_those_of_a_step_that_keeps_everything(tokens, width, hidden):
    from paper_1905_10988_b200.checkpointed_block import CheckpointedBlock
    block = CheckpointedBlock(tokens, width, hidden, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    dy = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    block.gamma.copy_(1 + 0.1 * torch.randn(width, generator=g, device="cuda"))
    block.beta.copy_(0.1 * torch.randn(width, generator=g, device="cuda"))
    grad = torch.full((block.gradient_size,), 9.0, device="cuda")
    y = block.forward(x, seed=1, worker=2)
    dx = block.backward(dy, grad)
    wy, wdx, want = _plain_step(block, x, dy)
    # bfloat16 keeps 8 bits, a checkpoint about 6 below a block's largest value; both errors are
    # random and average out in sums, so that a few percent of a gradient's norm bound them all
    def rel(a, b):
        return float((a.double() - b).norm() / b.norm())
    assert rel(y, wy) < 0.02 and rel(dx, wdx) < 0.03
    for name, (at, n) in block.slices.items():
        assert rel(grad[at:at + n].view_as(want[name]), want[name]) < 0.05, name
    # a second backward pass on top doubles the sums
    twice = grad.clone()
    block.backward(dy, twice, accumulate=True)
    for name, (at, n) in block.slices.items():
        assert torch.allclose(twice[at:at + n], 2 * grad[at:at + n], rtol=1e-5, atol=1e-5), name


def test_training_with_compressed_gradients_lowers_the_loss():
    from paper_1905_10988_b200.checkpointed_block import train
    losses, block = train(tokens=512, width=128, hidden=512, workers=3, steps=12, rate=0.05)
    assert np.isfinite(losses).all() and losses[-1] < 0.9 * losses[0]
    full = 2 * block.tokens * (block.width + 2 * block.hidden)
    assert block.checkpoint_bytes < 0.53 * full


def test_operators_are_captured_in_a_graph():
    import paper_1905_10988_b200 as nc
    t, w, n = 700, 1000, 300                          # two kernels and more a call, odd sizes
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(t, w, generator=g, device="cuda").bfloat16()
    dy = torch.randn(t, w, generator=g, device="cuda").bfloat16()
    dn = torch.randn(t, n, generator=g, device="cuda").bfloat16()
    u8, f32 = dict(dtype=torch.uint8, device="cuda"), dict(dtype=torch.float32, device="cuda")
    codes = torch.zeros(nc.nc_act8_code_bytes(t, w), **u8)
    scales = torch.zeros(nc.nc_act8_scale_bytes(t, w), **u8)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    rstd, dg, db = torch.empty(t, **f32), torch.empty(w, **f32), torch.empty(w, **f32)
    dw, dbias = torch.empty(n, w, **f32), torch.empty(n, **f32)
    size = max(nc.nc_layer_norm_workspace_bytes(t, w),
               nc.nc_act8_weight_grad_workspace_bytes(t, n, w))
    ws = torch.empty(size, **u8)
    B, F = nc.DTYPE_BF16, nc.DTYPE_F32

    def step():
        nc.nc_layer_norm_forward(x, B, t, w, w, None, None, F, 1e-5, y, w, None, rstd, codes, scales,
                                 nc.ROUND_NEAREST, 0, 0)
        nc.nc_act8_layer_norm_backward(dy, B, t, w, w, codes, scales, rstd, None, F, None, 0, dx, w,
                                       dg, db, False, ws, size)
        nc.nc_act8_weight_grad(dn, t, n, n, codes, scales, w, None, None, F, dw, F, w, dbias, False,
                               ws, size)

    step()
    torch.cuda.synchronize()
    outs = (y, dx, rstd, dg, db, dw, dbias)
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        step()
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for o in outs:
        o.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for o, v in zip(outs, want):
        assert torch.equal(o, v)
    # and the step's codes are those of the definition
    _, _, _, xh = ref.layer_norm(x.double().cpu().numpy(), None, None, 1e-5)
    kept = ref.decode(codes.cpu().numpy().reshape(t, -1),
                      scales.cpu().numpy()[:t * ref.pitch_of(w) // 32].reshape(t, -1), w)
    unit = np.ldexp(1.0, np.repeat(ref.scale_bytes(xh).astype(int), 32, 1)[:, :w] - 127)
    assert np.all(np.abs(kept - xh) <= 0.5001 * unit * 2)
