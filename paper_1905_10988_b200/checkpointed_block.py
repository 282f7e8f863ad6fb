"""A training step around the 8-bit activation checkpoints: a pre-norm feed-forward block with a
residual connection whose activations are kept in 8 bits, and whose gradients go to the compressors.

    y = x + W2 gelu(W1 norm(x) + b1) + b2

The forward pass keeps the normalised rows (written by the norm itself), the inputs of the
activation function and its outputs as checkpoints.  The backward pass reads the first and the
last as the inputs of the two linear layers, decoded inside the products of their weight gradients;
the norm's own backward pass reads the first one again.  All gradients are written into one fp32
vector, which nc_compress reads.

`python -m paper_1905_10988_b200.checkpointed_block` trains a block on the gradients of n simulated
workers, which are compressed and aggregated in every step, and prints the loss.
"""
from __future__ import annotations

import math

import torch

import paper_1905_10988_b200 as nc

EPS = 1e-5


class Checkpoint:
    """8-bit codes and scales of a rows x cols matrix."""

    def __init__(self, rows: int, cols: int, device):
        u8 = dict(dtype=torch.uint8, device=device)
        self.rows, self.cols = rows, cols
        self.codes = torch.empty(nc.nc_act8_code_bytes(rows, cols), **u8)
        self.scales = torch.empty(nc.nc_act8_scale_bytes(rows, cols), **u8)

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()

    def keep(self, x, rounding, seed, worker) -> None:
        """x: bfloat16 rows x cols."""
        ldx = _row_stride("x", x, self.rows, self.cols, torch.bfloat16, self.codes.device)
        nc.nc_act8_compress(x, nc.DTYPE_BF16, self.rows, self.cols, ldx, rounding, seed, worker,
                            self.codes, self.scales)

    def read(self):
        out = torch.empty(self.rows, self.cols, dtype=torch.bfloat16, device=self.codes.device)
        nc.nc_act8_decompress(self.codes, self.scales, self.rows, self.cols, out, nc.DTYPE_BF16,
                              self.cols)
        return out


def _row_stride(name: str, x, rows: int, cols: int, dtype, device) -> int:
    """The row stride of a matrix that the kernels may read as rows x cols of `dtype` on `device`;
    ValueError for any other.  The library sees an address and a stride only."""
    if x.dtype != dtype:
        raise ValueError("%s is %s, not %s" % (name, x.dtype, dtype))
    if tuple(x.shape) != (rows, cols):
        raise ValueError("%s has shape %s, not %s" % (name, tuple(x.shape), (rows, cols)))
    if (cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols):
        raise ValueError("%s has strides %s: rows of neighbouring values, one behind the other, are "
                         "needed" % (name, tuple(x.stride())))
    _on_device(name, x, device)
    return x.stride(0) if rows > 1 else cols


def _on_device(name: str, x, device) -> None:
    if x.device.type != "cuda" or x.device != device:
        raise ValueError("%s is on %s, not on the block's GPU (%s)" % (name, x.device, device))
    if x.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, which is not the current device" % (name, x.device))


def _gelu_and_slope(h):
    """gelu(h) = h * Phi(h) and its derivative, in fp32."""
    h = h.float()
    phi = 0.5 * (1 + torch.erf(h / math.sqrt(2)))
    return h * phi, phi + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)


class CheckpointedBlock:
    """Parameters (bfloat16) and the step's buffers for `tokens` rows of `width` columns."""

    NAMES = ("w1", "b1", "w2", "b2", "gamma", "beta")

    def __init__(self, tokens: int, width: int, hidden: int, seed: int = 0, device="cuda",
                 rounding: int = nc.ROUND_RANDOM):
        g = torch.Generator(device=device).manual_seed(seed)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.tokens, self.width, self.hidden, self.rounding = tokens, width, hidden, rounding
        self.w1 = (torch.randn(hidden, width, generator=g, device=device) / width ** 0.5).bfloat16()
        self.w2 = (torch.randn(width, hidden, generator=g, device=device) / hidden ** 0.5).bfloat16()
        self.b1, self.b2 = torch.zeros(hidden, **bf), torch.zeros(width, **bf)
        self.gamma, self.beta = torch.ones(width, **bf), torch.zeros(width, **bf)
        self.normed = Checkpoint(tokens, width, device)
        self.before = Checkpoint(tokens, hidden, device)      # the activation function's inputs
        self.after = Checkpoint(tokens, hidden, device)       # and outputs
        self.rstd = torch.empty(tokens, dtype=torch.float32, device=device)
        self.kept = False                                     # the checkpoints hold a forward pass
        # one fp32 vector for all gradients, every piece on a 32-byte boundary
        self.slices, at = {}, 0
        for name in self.NAMES:
            n = getattr(self, name).numel()
            self.slices[name] = (at, n)
            at += -(-n // 8) * 8
        self.gradient_size = at
        # what lies between the pieces: (begin, end)
        self.gaps = [(at + n, at + -(-n // 8) * 8) for at, n in self.slices.values() if n % 8]
        self.ws_bytes = max(nc.nc_layer_norm_workspace_bytes(tokens, width),
                            nc.nc_act8_weight_grad_workspace_bytes(tokens, hidden, width),
                            nc.nc_act8_weight_grad_workspace_bytes(tokens, width, hidden))
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    @property
    def checkpoint_bytes(self) -> int:
        return self.normed.nbytes + self.before.nbytes + self.after.nbytes

    def forward(self, x, seed: int = 0, worker: int = 0):
        """x: bfloat16 tokens x width.  seed and worker draw the checkpoints' rounding."""
        t, w = self.tokens, self.width
        ldx = _row_stride("x", x, t, w, torch.bfloat16, self.rstd.device)
        a = torch.empty(t, w, dtype=torch.bfloat16, device=x.device)
        nc.nc_layer_norm_forward(x, nc.DTYPE_BF16, t, w, ldx, self.gamma, self.beta, nc.DTYPE_BF16,
                                 EPS, a, w, None, self.rstd, self.normed.codes, self.normed.scales,
                                 self.rounding, seed, 3 * worker)
        h = torch.addmm(self.b1, a, self.w1.t())
        self.before.keep(h, self.rounding, seed, 3 * worker + 1)
        u = _gelu_and_slope(h)[0].bfloat16()
        self.after.keep(u, self.rounding, seed, 3 * worker + 2)
        self.kept = True
        return x + torch.addmm(self.b2, u, self.w2.t())

    def backward(self, dy, gradient, accumulate: bool = False):
        """dy: bfloat16 tokens x width.  Writes all parameters' gradients into the fp32 vector
        `gradient` (gradient_size entries; 0 between the pieces) and returns the gradient of x."""
        t, w, k = self.tokens, self.width, self.hidden
        lddy = _row_stride("dy", dy, t, w, torch.bfloat16, self.rstd.device)
        self._check_gradient(gradient)
        if not self.kept:
            raise RuntimeError("no forward pass has kept activations for this one")
        for begin, end in self.gaps:         # the compressors read them, and norms count them
            gradient[begin:end].zero_()
        piece = {name: gradient[at:at + n] for name, (at, n) in self.slices.items()}
        f32, bf16 = nc.DTYPE_F32, nc.DTYPE_BF16
        nc.nc_act8_weight_grad(dy, t, w, lddy, self.after.codes, self.after.scales, k, None,
                               None, bf16, piece["w2"], f32, k, piece["b2"], accumulate,
                               self.workspace, self.ws_bytes)
        slope = _gelu_and_slope(self.before.read())[1]
        dh = (torch.mm(dy, self.w2).float() * slope).bfloat16()
        nc.nc_act8_weight_grad(dh, t, k, k, self.normed.codes, self.normed.scales, w, self.gamma,
                               self.beta, bf16, piece["w1"], f32, w, piece["b1"], accumulate,
                               self.workspace, self.ws_bytes)
        da = torch.mm(dh, self.w1)
        dx = torch.empty(t, w, dtype=torch.bfloat16, device=dy.device)
        nc.nc_act8_layer_norm_backward(da, bf16, t, w, w, self.normed.codes, self.normed.scales,
                                       self.rstd, self.gamma, bf16, dy, lddy, dx, w, piece["gamma"],
                                       piece["beta"], accumulate, self.workspace, self.ws_bytes)
        return dx

    def _check_gradient(self, gradient) -> None:
        size = self.gradient_size
        if gradient.dtype != torch.float32 or gradient.dim() != 1 or gradient.numel() < size:
            raise ValueError("gradient is %s %s, not a torch.float32 vector of %d entries"
                             % (gradient.dtype, tuple(gradient.shape), size))
        if gradient.stride(0) != 1:
            raise ValueError("gradient has a stride of %d" % gradient.stride(0))
        _on_device("gradient", gradient, self.rstd.device)

    def apply(self, gradient, rate: float) -> None:
        """Plain gradient descent with the (aggregated) fp32 gradient vector."""
        for name, (at, n) in self.slices.items():
            p = getattr(self, name)
            p.copy_(p.float() - rate * gradient[at:at + n].view_as(p))


def train(tokens=2048, width=512, hidden=2048, workers=4, steps=40, rate=0.005, seed=0,
          device="cuda"):
    """The losses of `steps` steps of `workers` simulated workers on one device, whose gradients
    are exchanged as C_nat codes."""
    block = CheckpointedBlock(tokens, width, hidden, seed, device)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    xs = [torch.randn(tokens, width, generator=g, device=device).bfloat16() for _ in range(workers)]
    turn = torch.linalg.qr(torch.randn(width, width, generator=g, device=device))[0].bfloat16()
    goals = [torch.mm(x, turn) for x in xs]
    d = block.gradient_size
    f32, u8 = dict(dtype=torch.float32, device=device), dict(dtype=torch.uint8, device=device)
    gradients = [torch.zeros(d, **f32) for _ in range(workers)]
    exps = [torch.empty(nc.nc_exp_bytes(d), **u8) for _ in range(workers)]
    signs = [torch.empty(nc.nc_sign_bytes(d), **u8) for _ in range(workers)]
    total = torch.empty(d, **f32)
    losses = []
    for step in range(steps):
        loss = 0.0
        for i in range(workers):
            y = block.forward(xs[i], seed + step, i)
            diff = (y - goals[i]).float()
            loss = loss + (diff * diff).mean() / workers
            dy = (2 * diff / diff.numel() * width).bfloat16()
            block.backward(dy, gradients[i])
        nc.nc_compress_batch(gradients, d, seed + step, list(range(workers)), exps, signs, workers)
        nc.nc_aggregate(exps, signs, workers, d, total)
        block.apply(total, rate / workers)
        losses.append(loss)
    return [float(v) for v in losses], block


def main() -> None:
    losses, block = train()
    kept = block.checkpoint_bytes
    full = 2 * block.tokens * (block.width + 2 * block.hidden)
    print("loss %.4f -> %.4f over %d steps; activations kept: %.2f MB instead of %.2f MB"
          % (losses[0], losses[-1], len(losses), kept / 1e6, full / 1e6))


if __name__ == "__main__":
    main()
