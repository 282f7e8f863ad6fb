"""A small language model around the 8-bit activation checkpoints: tokens in, their loss out, and the
gradients of all parameters in one fp32 vector, which nc_compress reads.

    x = sqrt(width) * table[token]        nc_embedding_forward
    x = block(x), once for each block     CheckpointedBlock
    z = norm(x) table^T                   nc_layer_norm_forward
    loss = mean of lse(z) - z[target]     nc_linear_cross_entropy_forward: z is not kept

The blocks work on every token by itself (nothing mixes tokens), so the model learns which token follows which.
One table serves both ends: its gradient is written by nc_linear_cross_entropy_backward, and
nc_embedding_backward adds the rows of the batch's tokens to it.  A token below 0 is padding (its row is 0),
a target below 0 does not count.  apply() takes the aggregated gradient: the blocks' matrices move along
their orthogonalised gradients (nc_orthogonalize), everything else along the gradient itself.

`python -m paper_1905_10988_b200.token_model` trains a model on the gradients of n simulated workers,
which are compressed and aggregated in every step, and prints the loss.
"""
from __future__ import annotations

import torch

import paper_1905_10988_b200 as nc
from .checkpointed_block import EPS, CheckpointedBlock, _on_device

NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315) * 5      # a, b, c of each of five steps


def _token_bytes(name: str, t, count: int, device) -> int:
    """4 or 8, for a vector of `count` tokens that the kernels may read; ValueError for any other."""
    if t.dtype not in (torch.int32, torch.int64):
        raise ValueError("%s is %s, not torch.int32 or torch.int64" % (name, t.dtype))
    if tuple(t.shape) != (count,):
        raise ValueError("%s has shape %s, not %s" % (name, tuple(t.shape), (count,)))
    if count > 1 and t.stride(0) != 1:
        raise ValueError("%s has a stride of %d" % (name, t.stride(0)))
    _on_device(name, t, device)
    return t.element_size()


class TokenModel:
    """Parameters (bfloat16) and the step's buffers for `tokens` tokens at a time."""

    def __init__(self, tokens: int, vocabulary: int, width: int, hidden: int, blocks: int = 1,
                 seed: int = 0, device="cuda", rounding: int = nc.ROUND_RANDOM):
        g = torch.Generator(device=device).manual_seed(seed)
        bf = dict(dtype=torch.bfloat16, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.tokens, self.vocabulary, self.width = tokens, vocabulary, width
        self.table = (torch.randn(vocabulary, width, generator=g, device=device)
                      / width ** 0.5).bfloat16()
        self.scale = width ** 0.5
        self.blocks = [CheckpointedBlock(tokens, width, hidden, seed + 1 + i, device, rounding)
                       for i in range(blocks)]
        self.gamma, self.beta = torch.ones(width, **bf), torch.zeros(width, **bf)
        # one fp32 vector for all gradients: the blocks' in turn, then these; every piece on a
        # 32-byte boundary
        self.block_slices, self.slices, at = [], {}, 0
        for b in self.blocks:
            self.block_slices.append((at, b.gradient_size))
            at += b.gradient_size
        for name in ("table", "gamma", "beta"):
            n = getattr(self, name).numel()
            self.slices[name] = (at, n)
            at += -(-n // 8) * 8
        self.gradient_size = at
        self.gaps = [(a + n, a + -(-n // 8) * 8) for a, n in self.slices.values() if n % 8]
        # what the forward pass leaves for the backward pass
        self.ids = self.targets = None
        self.last, self.normed = torch.empty(tokens, width, **bf), torch.empty(tokens, width, **bf)
        self.mean, self.rstd = torch.empty(tokens, **f32), torch.empty(tokens, **f32)
        self.loss, self.lse = torch.empty(tokens, **f32), torch.empty(tokens, **f32)
        self.weight = torch.empty(tokens, **f32)
        sizes = (tokens, width, vocabulary)
        shapes = {(b.hidden, width) for b in self.blocks} | {(width, b.hidden) for b in self.blocks}
        self.ws_bytes = max([nc.nc_linear_cross_entropy_forward_workspace_bytes(*sizes),
                             nc.nc_linear_cross_entropy_backward_workspace_bytes(*sizes),
                             nc.nc_embedding_backward_workspace_bytes(tokens, vocabulary, width),
                             nc.nc_layer_norm_workspace_bytes(tokens, width)]
                            + [nc.nc_orthogonalize_workspace_bytes(1, *s) for s in shapes])
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    def forward(self, ids, targets, seed: int = 0, worker: int = 0):
        """ids, targets: `tokens` int32 or int64 tokens each.  -> the mean loss over the targets that
        count, a tensor of one value.  seed and worker draw the checkpoints' rounding."""
        t, w, v, bf16 = self.tokens, self.width, self.vocabulary, nc.DTYPE_BF16
        device = self.lse.device
        id_bytes = _token_bytes("ids", ids, t, device)
        target_bytes = _token_bytes("targets", targets, t, device)
        x = torch.empty(t, w, dtype=torch.bfloat16, device=device)
        nc.nc_embedding_forward(ids, id_bytes, t, self.table, bf16, v, w, w, self.scale, x, bf16, w)
        for i, b in enumerate(self.blocks):
            x = b.forward(x, seed, worker * len(self.blocks) + i)
        self.last.copy_(x)
        nc.nc_layer_norm_forward(self.last, bf16, t, w, w, self.gamma, self.beta, bf16, EPS,
                                 self.normed, w, self.mean, self.rstd, None, None,
                                 nc.ROUND_NEAREST, 0, 0)
        nc.nc_linear_cross_entropy_forward(self.normed, bf16, t, w, w, self.table, v, w, targets,
                                           target_bytes, 1.0, self.loss, self.lse, self.workspace,
                                           self.ws_bytes)
        counts = (targets >= 0).float()
        torch.div(counts, counts.sum().clamp(min=1.0), out=self.weight)
        self.ids, self.targets = ids, targets
        return (self.loss * self.weight).sum()

    def backward(self, gradient) -> None:
        """Writes the gradients of the mean loss into the fp32 vector `gradient` (gradient_size
        entries; 0 between the pieces).  ids and targets of the forward pass are read again."""
        if self.ids is None:
            raise RuntimeError("no forward pass has kept activations for this one")
        t, w, v, bf16, f32 = self.tokens, self.width, self.vocabulary, nc.DTYPE_BF16, nc.DTYPE_F32
        self._check_gradient(gradient)
        for begin, end in self.gaps:
            gradient[begin:end].zero_()
        piece = {name: gradient[at:at + n] for name, (at, n) in self.slices.items()}
        dx = torch.empty(t, w, dtype=torch.bfloat16, device=gradient.device)
        nc.nc_linear_cross_entropy_backward(
            self.normed, bf16, t, w, w, self.table, v, w, self.targets, self.targets.element_size(),
            1.0, self.lse, self.weight, None, dx, w, piece["table"], f32, w, False, self.workspace,
            self.ws_bytes)
        dy, dx = dx, torch.empty_like(dx)
        nc.nc_layer_norm_backward(dy, bf16, t, w, w, self.last, w, self.mean, self.rstd, self.gamma,
                                  bf16, None, 0, dx, w, piece["gamma"], piece["beta"], False,
                                  self.workspace, self.ws_bytes)
        for b, (at, n) in reversed(list(zip(self.blocks, self.block_slices))):
            dx = b.backward(dx, gradient[at:at + n])
        nc.nc_embedding_backward(self.ids, self.ids.element_size(), t, dx, bf16, w, w, self.scale, v,
                                 piece["table"], f32, w, True, self.workspace, self.ws_bytes)

    def _check_gradient(self, gradient) -> None:
        if gradient.dtype != torch.float32 or tuple(gradient.shape) != (self.gradient_size,):
            raise ValueError("gradient is %s %s, not a torch.float32 vector of %d entries"
                             % (gradient.dtype, tuple(gradient.shape), self.gradient_size))
        if gradient.stride(0) != 1:
            raise ValueError("gradient has a stride of %d" % gradient.stride(0))
        _on_device("gradient", gradient, self.lse.device)

    def apply(self, gradient, rate: float, matrix_rate: float) -> None:
        """One step along the (aggregated) gradient, an fp32 vector of gradient_size entries: the blocks'
        matrices by matrix_rate times their orthogonalised gradients, which have singular values near 1
        whatever the gradient's size, the rest by rate times the gradient."""
        self._check_gradient(gradient)
        for b, (at, n) in zip(self.blocks, self.block_slices):
            for name, (begin, size) in b.slices.items():
                p, g = getattr(b, name), gradient[at + begin:at + begin + size]
                if name in ("w1", "w2"):
                    rows, cols = p.shape
                    step = torch.empty(rows, cols, dtype=torch.float32, device=p.device)
                    nc.nc_orthogonalize(g, nc.DTYPE_F32, 1, rows, cols, cols, size, NEWTON_SCHULZ,
                                        len(NEWTON_SCHULZ) // 3, 1e-7,
                                        max(1.0, rows / cols) ** 0.5, step, nc.DTYPE_F32, cols, size,
                                        self.workspace, self.ws_bytes)
                    p.copy_(p.float() - matrix_rate * step)
                else:
                    p.copy_(p.float() - rate * g.view_as(p))
        for name, (at, n) in self.slices.items():
            p = getattr(self, name)
            p.copy_(p.float() - rate * gradient[at:at + n].view_as(p))


def train(tokens=2048, vocabulary=8192, width=512, hidden=2048, blocks=2, workers=4, steps=40, rate=2.0,
          matrix_rate=0.02, seed=0, device="cuda"):
    """The losses of `steps` steps of `workers` simulated workers on one device, whose gradients are
    exchanged as C_nat codes.  Every token has one successor, and a few are padding."""
    model = TokenModel(tokens, vocabulary, width, hidden, blocks, seed, device)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    follows = torch.randperm(vocabulary, generator=g, device=device)
    d = model.gradient_size
    u8 = dict(dtype=torch.uint8, device=device)
    gradients = [torch.zeros(d, dtype=torch.float32, device=device) for _ in range(workers)]
    exps = [torch.empty(nc.nc_exp_bytes(d), **u8) for _ in range(workers)]
    signs = [torch.empty(nc.nc_sign_bytes(d), **u8) for _ in range(workers)]
    total = torch.empty(d, dtype=torch.float32, device=device)
    losses = []
    for step in range(steps):
        loss = 0.0
        for i in range(workers):
            u = torch.rand(tokens, generator=g, device=device)
            ids = (vocabulary ** u).long().clamp(max=vocabulary) - 1       # few tokens are frequent
            targets = follows[ids]
            ids[-tokens // 16:] = targets[-tokens // 16:] = -1
            loss = loss + model.forward(ids, targets, seed + step, i) / workers
            model.backward(gradients[i])
        nc.nc_compress_batch(gradients, d, seed + step, list(range(workers)), exps, signs, workers)
        nc.nc_aggregate(exps, signs, workers, d, total)
        model.apply(total, rate / workers, matrix_rate)
        losses.append(loss)
    return [float(v) for v in losses], model


def main() -> None:
    losses, model = train()
    print("loss %.4f -> %.4f over %d steps; logits that were not kept: %.2f MB a worker and step"
          % (losses[0], losses[-1], len(losses), 4e-6 * model.tokens * model.vocabulary))


if __name__ == "__main__":
    main()
