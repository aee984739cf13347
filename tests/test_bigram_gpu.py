"""The lookup, the table's gradient, the clipped norm and the optimizers run together (the package's small language
model): its gradient against autograd in 64 bits, and what it learns."""
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


def test_gradient_of_the_tied_table_against_autograd():
    """In binary32 through products of 40 and 200 terms: 2^-24 times those, a few operations a term, of the largest
    gradient (2e-5 is eight times 256 u)."""
    device = torch.device("cuda", 0)
    vocab, dim = 200, 40
    model, batch = Bigram(vocab, dim, 64, device, seed=1), Corpus(vocab, 2, device).batch(4, 16, 3)
    model.x[-dim:] = 0.1
    g = torch.empty_like(model.x)
    loss = model.gradient(batch, g)
    x = model.x.double().requires_grad_()
    E, M, b = x.split(model.sizes)
    E, M = E.view(vocab, dim), M.view(dim, dim)
    h = E[batch[:, :-1].reshape(-1)] * dim ** 0.5 @ M + b
    want = torch.nn.functional.cross_entropy(h @ E.t(), batch[:, 1:].reshape(-1))
    want.backward()
    torch.backends.cuda.matmul.allow_tf32 = False
    scale = float(x.grad.abs().max())
    assert abs(float(loss) - float(want.detach())) <= 2e-5 * float(want.detach())
    assert float((g.double() - x.grad).abs().max()) <= 2e-5 * scale


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8", "round"])
def test_every_optimizer_learns(optimizer):
    """Four likely successors a token: the loss starts at log 512 and falls well below half of it (log 4 is the
    least)."""
    losses = train(optimizer, steps=150)
    assert abs(losses[0] - np.log(512)) < 0.1
    assert np.mean(losses[-10:]) < 0.5 * np.log(512)


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8", "round"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_gradient_that_is_not_finite_does_not_stay(monkeypatch, optimizer, bad):
    """Every worker's gradient of the fourth step holds a value that is not finite: the training goes on and learns."""
    calls, gradient = [], Bigram.gradient

    def poisoned(self, batch, g):
        loss = gradient(self, batch, g)
        calls.append(1)
        if 3 * 4 < len(calls) <= 4 * 4:
            g[5] = bad
        return loss

    monkeypatch.setattr(Bigram, "gradient", poisoned)
    losses = train(optimizer, steps=60)
    assert len(calls) == 60 * 4 and np.isfinite(losses).all()
    assert np.mean(losses[-5:]) < 0.9 * np.log(512)
