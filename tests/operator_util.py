"""Helpers of the tests of the embedding, the cross entropy and the orthogonalised update."""
import torch

import paper_1905_10988_b200 as nc

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"f32": nc.DTYPE_F32, "bf16": nc.DTYPE_BF16, "f16": nc.DTYPE_F16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # half a step, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}    # and of subnormal numbers


class Placed:
    """A matrix (or several at a distance) on the GPU with rows `gap` elements longer than needed, from
    element `offset` of its memory on, between bands that a call must leave alone."""

    def __init__(self, shape, kind, layout="whole", fill=None):
        *batch, rows, cols = shape
        self.batch = batch[0] if batch else 1
        gap, offset = {"whole": (0, 64), "gap": (16 - cols % 16, 64), "any": (3, 65)}[layout]
        self.ld = cols + gap
        self.distance = rows * self.ld + (5 if layout == "any" else 16 if layout == "gap" else 0)
        need = offset + self.batch * self.distance + 64
        self.memory = torch.full((need,), float("nan"), dtype=TYPES[kind], device="cuda")
        self.memory.fill_(-77.0)
        self.before = self.memory.clone()
        stride = (self.distance, self.ld, 1) if batch else (self.ld, 1)
        self.view = self.memory.as_strided(shape, stride, offset)
        if fill is not None:
            self.view.copy_(fill)

    def untouched(self):
        """Nothing but the matrix has changed."""
        inside = torch.zeros_like(self.memory, dtype=torch.bool)
        inside.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(True)
        return bool((self.memory == self.before)[~inside].all())


def workspace(size):
    """A workspace filled with NaN, and bands around it."""
    ws = torch.full((size + 512,), 255, dtype=torch.uint8, device="cuda")
    return ws, ws[256:256 + size]


def status(call):
    try:
        call()
    except nc.NatcompError as e:
        return nc.status_string(e.status)
    return "NC_OK"


def address():
    """Memory for calls that must be refused: real on a GPU, a number that nothing reads without one."""
    if torch.cuda.is_available():
        buf = torch.zeros(2 << 20, dtype=torch.uint8, device="cuda")
        return buf, (buf.data_ptr() + 255) & ~255
    return None, 1 << 20


def within(got, want, tol):
    """The largest excess over the tolerance, as a ratio of it."""
    off = (got.double() - want).abs()
    return bool((off <= tol).all()), float((off / tol).max()) if off.numel() else 0.0
