"""Layer norm, the gated recurrence and dropout run together with the lookup, the clipped norm and the optimizers: the package's
small language model with blocks, its gradient against autograd in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2205_14473_gb300.bigram import Bigram, Corpus, train

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)


def _loss(model, x, batch, masks):
    """The model's loss in 64 bits, differentiable in the flat vector x."""
    E, M, b, *rest = x.split(model.sizes)
    E, M = E.view(model.vocab, model.dim), M.view(model.dim, model.dim)
    e = E[batch[:, :-1]] * model.scale
    for (w, c, A, a, O), mask in zip(model._blocks(rest), masks):
        d = e - e.mean(-1, keepdim=True)
        y = d * (d.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w + c
        z, v = (y @ A + a).split(model.dim, -1)
        f, state, rows = torch.sigmoid(z), torch.zeros_like(z[:, 0]), []
        for t in range(z.shape[1]):
            state = f[:, t] * state + (1 - f[:, t]) * v[:, t]
            rows.append(state)
        e = e + torch.stack(rows, 1) @ O * mask
    h = e.reshape(-1, model.dim) @ M + b
    return torch.nn.functional.cross_entropy(h @ E.t(), batch[:, 1:].reshape(-1))


@pytest.mark.parametrize("blocks,dropout", [(1, 0.0), (2, 0.1), (3, 0.5)])
def test_gradient_of_the_blocks_against_autograd(blocks, dropout):
    """In binary32: of up to three blocks the products' sums of 80 terms, the norm's of 40 and 16 rows of the recurrence with five
    roundings each, and of the head sums of 40 and 200 terms: below 2,000 roundings one behind another, each of at most u = 2^-24
    of the largest gradient."""
    torch.backends.cuda.matmul.allow_tf32 = False
    device = torch.device("cuda", 0)
    vocab, dim, shape = 200, 40, (4, 16)
    model, batch = Bigram(vocab, dim, 64, device, seed=1, blocks=blocks, dropout=dropout), Corpus(vocab, 2, device).batch(*shape, 3)
    g = torch.full_like(model.x, float("nan"))
    model.draws = 7
    loss = model.gradient(batch, g)
    assert model.draws == 7 + blocks
    ones = torch.ones(*shape, dim, device=device)
    masks = [model.drop(ones, 7 + k).double() for k in range(blocks)]  # 1 / (1 - p) or 0
    x = model.x.double().requires_grad_()
    want = _loss(model, x, batch, masks)
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 2000 * 2.0 ** -24 * float(want.detach())
    assert float((g.double() - x.grad).abs().max()) <= 2000 * 2.0 ** -24 * float(x.grad.abs().max())


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8", "round"])
def test_blocks_run_under_every_optimizer(optimizer):
    losses = train(optimizer, steps=12, blocks=2, dropout=0.1, workers=2)
    assert len(losses) == 12 and np.isfinite(losses).all() and abs(losses[0] - np.log(512)) < 0.5


def test_a_model_without_blocks_is_as_it_was():
    device = torch.device("cuda", 0)
    a, b = Bigram(50, 8, 64, device, seed=3), Bigram(50, 8, 64, device, seed=3, blocks=2, dropout=0.1)
    assert torch.equal(a.x, b.x[:a.x.numel()]) and a.sizes == b.sizes[:3]
