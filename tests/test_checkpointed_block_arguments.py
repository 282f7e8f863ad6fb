"""What CheckpointedBlock refuses: the library reads addresses and strides only, so a tensor of another
type, shape, stride or device has to be refused before any call.  No GPU is needed: a refusal comes
before the first launch, and tensors that are not on a GPU are themselves refused."""
import pytest
import torch

from paper_1905_10988_b200.checkpointed_block import CheckpointedBlock, Checkpoint

T, W, H = 6, 20, 12


def block():
    return CheckpointedBlock(T, W, H, device="cpu")


def bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


BAD = [
    ("type", lambda: torch.zeros(T, W), "float32"),
    ("half", lambda: torch.zeros(T, W, dtype=torch.float16), "float16"),
    ("short last batch", lambda: bf(T - 1, W), "shape"),
    ("longer", lambda: bf(T + 1, W), "shape"),
    ("narrow", lambda: bf(T, W - 1), "shape"),
    ("one dimension", lambda: bf(T * W), "shape"),
    ("every second column", lambda: bf(T, 2 * W)[:, ::2], "strides"),
    ("transposed", lambda: bf(W, T).t(), "strides"),
    ("one row for all", lambda: bf(1, W).expand(T, W), "strides"),
    ("overlapping rows", lambda: bf(T * W).as_strided((T, W), (W - 1, 1)), "strides"),
    ("host memory", lambda: bf(T, W), "cpu"),
]


@pytest.mark.parametrize("name,make,says", BAD, ids=[b[0] for b in BAD])
def test_rows_are_checked_before_a_call(name, make, says):
    b = block()
    with pytest.raises(ValueError, match=says):
        b.forward(make())
    b.kept = True
    with pytest.raises(ValueError, match=says):
        b.backward(make(), torch.zeros(b.gradient_size))
    with pytest.raises(ValueError, match=says):
        Checkpoint(T, W, "cpu").keep(make(), 0, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("make,says", [
    (lambda n: torch.zeros(n - 1, device="cuda"), "gradient"),
    (lambda n: torch.zeros(n, device="cuda").double(), "float64"),
    (lambda n: torch.zeros(1, n, device="cuda"), "gradient"),
    (lambda n: torch.zeros(2 * n, device="cuda")[::2], "stride"),
    (lambda n: torch.zeros(n), "cpu"),
])
def test_gpu_gradient_vector_is_checked_before_a_call(make, says):
    b = CheckpointedBlock(T, W, H)
    x = bf(T, W).cuda()
    b.forward(x)
    with pytest.raises(ValueError, match=says):
        b.backward(x, make(b.gradient_size))


@pytest.mark.gpu
def test_gpu_no_backward_pass_without_a_forward_pass():
    b = CheckpointedBlock(T, W, H)
    with pytest.raises(RuntimeError, match="forward"):
        b.backward(bf(T, W).cuda(), torch.zeros(b.gradient_size, device="cuda"))


@pytest.mark.gpu
def test_gpu_views_and_single_tokens_give_what_whole_rows_give():
    g = torch.Generator(device="cuda").manual_seed(1)
    for tokens in (T, 1):
        b = CheckpointedBlock(tokens, W, H)
        wide = torch.randn(tokens, 3 * W, generator=g, device="cuda").bfloat16()
        x, dy = wide[:, W:2 * W], wide[:, 2 * W:]
        if tokens == 1:      # a row stride that no second row gives a meaning to
            x, dy = (v.as_strided((1, W), (1, 1)) for v in (x, dy))
        outs = []
        for u, v in ((x, dy), (x.clone().contiguous(), dy.clone().contiguous())):
            grad = torch.zeros(b.gradient_size, device="cuda")
            outs.append((b.forward(u), b.backward(v, grad), grad))
        assert all(torch.equal(p, q) for p, q in zip(*outs))


@pytest.mark.gpu
@pytest.mark.parametrize("width,hidden", [(100, 50), (20, 13), (64, 64)])
def test_gpu_every_entry_of_the_gradient_vector_is_written(width, hidden):
    # what lies between the pieces goes to the compressors as well: an inf or NaN there would set
    # the norm of a whole bucket
    b = CheckpointedBlock(T, width, hidden)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(T, width, generator=g, device="cuda").bfloat16()
    b.forward(x)
    between = torch.ones(b.gradient_size, dtype=torch.bool, device="cuda")
    for at, n in b.slices.values():
        between[at:at + n] = False
    for accumulate in (False, True):
        grad = torch.full((b.gradient_size + 3,), float("nan"), device="cuda")
        if accumulate:
            grad[:b.gradient_size][~between] = 0.0
        b.backward(x, grad, accumulate)
        assert bool(torch.isfinite(grad[:b.gradient_size]).all())
        assert not bool(grad[:b.gradient_size][between].any())
        assert bool(torch.isnan(grad[b.gradient_size:]).all())
