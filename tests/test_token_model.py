"""The embedding, the checkpointed blocks, the loss and the update together: a step's gradients against a
64-bit step that keeps everything, what is refused, and a few steps with compressed gradients."""
import pytest
import torch


def _plain(model, ids, targets):
    """Loss and gradients of the same model in float64 with nothing kept in 8 bits."""
    leaves = {n: getattr(model, n).double().requires_grad_() for n in ("table", "gamma", "beta")}
    x = model.scale * leaves["table"][ids.clamp(min=0)] * (ids >= 0).double()[:, None]

    def norm(x, gamma, beta):
        c = x - x.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma + beta

    blocks = []
    for b in model.blocks:
        p = {n: getattr(b, n).double().requires_grad_() for n in b.NAMES}
        h = norm(x, p["gamma"], p["beta"]) @ p["w1"].t() + p["b1"]
        u = 0.5 * h * (1 + torch.erf(h / 2 ** 0.5))
        x = x + u @ p["w2"].t() + p["b2"]
        blocks.append(p)
    z = norm(x, leaves["gamma"], leaves["beta"]) @ leaves["table"].t()
    there = targets >= 0
    loss = torch.nn.functional.cross_entropy(z[there], targets[there])
    loss.backward()
    return loss.detach(), {n: v.grad for n, v in leaves.items()}, [{n: v.grad for n, v in p.items()} for p in blocks]


def _batch(model, seed, padded):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, model.vocabulary, (model.tokens,), generator=g, device="cuda")
    targets = torch.randint(0, model.vocabulary, (model.tokens,), generator=g, device="cuda")
    if padded:
        ids[-padded:] = -1
        targets[-padded - 5:] = -1
    return ids, targets


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocabulary,width,hidden,blocks,padded",
                         [(300, 1000, 96, 200, 1, 40), (700, 777, 128, 256, 2, 0), (64, 50, 33, 40, 1, 3)])
def test_gradients_are_near_those_of_a_step_that_keeps_everything(tokens, vocabulary, width, hidden, blocks,
                                                                  padded):
    from paper_1905_10988_b200.token_model import TokenModel
    model = TokenModel(tokens, vocabulary, width, hidden, blocks, seed=3)
    ids, targets = _batch(model, 4, padded)
    grad = torch.full((model.gradient_size,), 9.0, device="cuda")
    loss = model.forward(ids, targets.int(), seed=1, worker=2)
    model.backward(grad)
    want, leaves, per_block = _plain(model, ids, targets)
    # bfloat16 keeps 8 bits, a checkpoint about 6 below a block's largest value; both errors are random
    # and average out in sums, so that a few percent of a gradient's norm bound them all
    assert abs(float(loss) - float(want)) < 0.02 * float(want)

    def rel(got, want):
        return float((got.double() - want).norm() / want.norm())

    for name, (at, n) in model.slices.items():
        assert rel(grad[at:at + n].view_as(leaves[name]), leaves[name]) < 0.05, name
    for b, p, (begin, _) in zip(model.blocks, per_block, model.block_slices):
        for name, (at, n) in b.slices.items():
            assert rel(grad[begin + at:begin + at + n].view_as(p[name]), p[name]) < 0.05, name
    for begin, end in model.gaps:
        assert bool((grad[begin:end] == 0).all())


@pytest.mark.gpu
def test_a_step_is_captured_and_replayed():
    from paper_1905_10988_b200.token_model import TokenModel
    model = TokenModel(256, 500, 64, 128, 2, seed=5)
    ids, targets = _batch(model, 6, 20)
    grad, again = (torch.zeros(model.gradient_size, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.forward(ids, targets)
        model.backward(grad)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = model.forward(ids, targets)
        model.backward(again)
    for seed in (6, 7):
        new = _batch(model, seed, 20)
        ids.copy_(new[0])
        targets.copy_(new[1])
        graph.replay()
        want = model.forward(ids, targets)
        model.backward(grad)
        torch.cuda.synchronize()
        assert torch.equal(again, grad) and float(loss) == float(want)


@pytest.mark.gpu
def test_steps_with_compressed_gradients_run_and_keep_the_parameters_finite():
    from paper_1905_10988_b200.token_model import train
    losses, model = train(tokens=256, vocabulary=700, width=64, hidden=128, blocks=2, workers=3, steps=4)
    assert len(losses) == 4 and all(v == v and abs(v) < 1e4 for v in losses)
    for p in [model.table, model.gamma] + [b.w1 for b in model.blocks] + [b.w2 for b in model.blocks]:
        assert bool(p.float().isfinite().all())


@pytest.mark.gpu
def test_arguments_are_checked():
    from paper_1905_10988_b200.token_model import TokenModel
    model = TokenModel(32, 40, 16, 32)
    ids, targets = _batch(model, 1, 0)
    grad = torch.zeros(model.gradient_size, device="cuda")
    with pytest.raises(RuntimeError):
        model.backward(grad)
    for a, b in ((ids.float(), targets), (ids[:-1], targets), (ids, targets.cpu()), (ids, targets.short()),
                 (torch.zeros(64, dtype=torch.long, device="cuda")[::2], targets), (ids.view(4, 8), targets)):
        with pytest.raises(ValueError):
            model.forward(a, b)
    model.forward(ids, targets)
    for g in (grad[:-1], grad.double(), grad.cpu(), torch.zeros(2 * grad.numel(), device="cuda")[::2]):
        with pytest.raises(ValueError):
            model.backward(g)
