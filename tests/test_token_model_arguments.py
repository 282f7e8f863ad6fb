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
