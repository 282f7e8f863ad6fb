"""What TokenModel.apply refuses and what it does: the library reads addresses only, so a gradient of another
type, length, stride or device has to be refused before a parameter has moved.  The refusals need no GPU."""
import numpy as np
import pytest
import torch

from operator_util import HALF, U
from paper_1905_10988_b200.token_model import NEWTON_SCHULZ, TokenModel

SIZES = dict(tokens=16, vocabulary=30, width=24, hidden=40, blocks=2)


def parameters(model):
    named = [(n, getattr(model, n)) for n in ("table", "gamma", "beta")]
    for i, b in enumerate(model.blocks):
        named += [("%s of block %d" % (n, i), getattr(b, n)) for n in b.NAMES]
    return named


BAD = [
    ("shorter", lambda n, dev: torch.ones(n - 1, device=dev), "gradient"),
    ("longer", lambda n, dev: torch.ones(n + 8, device=dev), "gradient"),
    ("bfloat16", lambda n, dev: torch.ones(n, dtype=torch.bfloat16, device=dev), "bfloat16"),
    ("binary64", lambda n, dev: torch.ones(n, dtype=torch.float64, device=dev), "float64"),
    ("a row", lambda n, dev: torch.ones(1, n, device=dev), "gradient"),
    ("every second one", lambda n, dev: torch.ones(2 * n, device=dev)[::2], "stride"),
    ("one for all", lambda n, dev: torch.ones(1, device=dev).expand(n), "stride"),
    ("host memory", lambda n, dev: torch.ones(n), "cpu"),
]


def refused(model, make, says):
    before = [p.clone() for _, p in parameters(model)]
    with pytest.raises(ValueError, match=says):
        model.apply(make(model.gradient_size, model.table.device), 0.1, 0.1)
    for (name, p), old in zip(parameters(model), before):
        assert torch.equal(p, old), name


@pytest.mark.parametrize("name,make,says", BAD, ids=[b[0] for b in BAD])
def test_apply_refuses(name, make, says):
    refused(TokenModel(**SIZES, device="cpu"), make, says)


@pytest.mark.gpu
@pytest.mark.parametrize("name,make,says", BAD, ids=[b[0] for b in BAD])
def test_apply_refuses_on_the_gpu(name, make, says):
    refused(TokenModel(**SIZES), make, says)


@pytest.mark.gpu
def test_apply_moves_every_parameter_by_its_own_formula():
    model = TokenModel(**SIZES, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    gradient = 1e-3 * torch.randn(model.gradient_size, generator=g, device="cuda")
    rate, matrix_rate = 30.0, 0.4
    pieces = [(n, getattr(model, n), at, size) for n, (at, size) in model.slices.items()]
    for b, (begin, _) in zip(model.blocks, model.block_slices):
        pieces += [(n, getattr(b, n), begin + at, size) for n, (at, size) in b.slices.items()]
    assert len(pieces) == 3 + 6 * len(model.blocks)
    want, slack = [], []
    for name, p, at, size in pieces:
        d = gradient[at:at + size].double().view_as(p)
        if name in ("w1", "w2"):
            x = d / (d.norm() + 1e-7)
            x = x.t() if p.shape[0] > p.shape[1] else x
            for a, b, c in np.float32(NEWTON_SCHULZ).astype(float).reshape(-1, 3):
                y = x @ x.t()
                x = a * x + (b * y + c * (y @ y)) @ x
            x = x.t() if p.shape[0] > p.shape[1] else x
            step = matrix_rate * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * x
            slack.append(8 * 2.0 ** -11 * float(step.norm()))          # the update's own error
        else:
            step = rate * d
            slack.append(4 * U * float(step.norm()))
        want.append(p.double() - step)
        # rounded to bfloat16 once, and the sums in binary32 before; a step left out, or of the wrong sign, is off
        # by its norm at least
        slack[-1] += (HALF["bf16"] + 4 * U) * float(want[-1].norm())
        assert float(step.norm()) > 3 * slack[-1], name
    model.apply(gradient, rate, matrix_rate)
    for (name, p, _, _), w, s in zip(pieces, want, slack):
        off = float((p.double() - w).norm())
        assert off <= s, (name, off)
