"""A small language model trained through this package's operators, with or without communication.

The model predicts the next token from the current one through a table E (vocab x dim) that is used twice, as the
input embedding and, tied, as the output head:  logits = h E^T,  h = s E[token] M + b.  Its parameters are one flat
vector [E, M, b], as EARound takes it.  A worker's step is

    e = table.lookup(tokens, E)             the embedding lookup (scale s)
    h, the logits, their cross-entropy and its gradient     (torch)
    dE = dlogits^T h                        the head's part of the table's gradient     (torch)
    table.grad(tokens, de, out=dE, accumulate=True)         the lookup's part, added to it
    clip = norm([g])                        the gradient's norm and clipping factor

and the parameters move either by AdamW on the clipped mean gradient (32- or 8-bit states), or by a round of
Efficient-Adam, in which every worker compresses its clipped gradient's Adam step.  A gradient that is not finite is not
used: AdamW skips the step, a worker of the round takes part with a gradient of zeros.

With blocks, the model sees more than the current token: between lookup and head stand residual blocks of a gated linear
recurrence, e <- e + dropout(scan(z, v) O) with [z, v] = layernorm(e) A + a, whose parameters (the norm's weight and bias, A, a,
O) follow in the flat vector:

    y, stats = norm.forward(e, w, b)        z, v = (y A + a)    (torch)
    h, _ = scan.forward(z, v)               e = drop(h O, counter, residual=e)

and back the same way, every operator by its own gradient.

    python -m paper_2205_14473_gb300.bigram --optimizer adamw8
    python -m paper_2205_14473_gb300.bigram --optimizer round --workers 4
    python -m paper_2205_14473_gb300.bigram --optimizer adamw --blocks 2 --dropout 0.1
"""
from __future__ import annotations

import argparse

import torch

import paper_2205_14473_gb300 as ea
from paper_2205_14473_gb300 import workloads as W


class Corpus:
    """Sequences of a random Markov chain over `vocab` tokens, each with a handful of likely successors."""

    def __init__(self, vocab: int, seed: int, device):
        gen = torch.Generator().manual_seed(seed)
        self.next = torch.randint(vocab, (vocab, 4), generator=gen).to(device)
        self.vocab, self.device = vocab, device

    def batch(self, sequences: int, length: int, seed: int):
        """[sequences, length + 1] tokens."""
        gen = torch.Generator(device=self.device).manual_seed(seed)
        out = [torch.randint(self.vocab, (sequences,), generator=gen, device=self.device)]
        for _ in range(length):
            pick = torch.randint(4, (sequences,), generator=gen, device=self.device)
            out.append(self.next[out[-1], pick])
        return torch.stack(out, 1)


class Bigram:
    """The parameters (one flat vector) and a worker's gradient."""

    def __init__(self, vocab: int, dim: int, tokens: int, device, seed: int = 0, blocks: int = 0, dropout: float = 0.0):
        if dropout and not blocks:
            raise ValueError("dropout is in the blocks, and there are none")
        self.vocab, self.dim, self.scale = vocab, dim, dim ** 0.5
        self.sizes = [vocab * dim, dim * dim, dim] + [dim, dim, 2 * dim * dim, 2 * dim, dim * dim] * blocks
        gen = torch.Generator(device=device).manual_seed(seed)
        self.x = torch.zeros(sum(self.sizes), device=device)
        table, turn, self.bias, *rest = self.x.split(self.sizes)
        self.E, self.M = table.view(vocab, dim), turn.view(dim, dim)
        self.E.normal_(0.0, 0.02, generator=gen)
        self.M.normal_(0.0, dim ** -0.5, generator=gen)
        self.table = ea.Embedding(vocab, dim, max_tokens=tokens, scale=self.scale)
        self.blocks = self._blocks(rest)
        self.draws = 0  # of the dropout's masks
        if blocks:
            self.norm, self.scan, self.drop = ea.LayerNorm(dim, max_rows=tokens), ea.GatedScan(dim), ea.Dropout(dropout, seed=seed + 1)
            for w, _, A, a, O in self.blocks:
                w.fill_(1.0)
                A.normal_(0.0, dim ** -0.5, generator=gen)
                a[:dim] = 1.0  # gates that start by remembering
                O.normal_(0.0, dim ** -0.5, generator=gen)

    def _blocks(self, pieces):
        d = self.dim
        return [(w, b, A.view(d, 2 * d), a, O.view(d, d)) for w, b, A, a, O in zip(*[iter(pieces)] * 5)]

    def gradient(self, batch, g) -> torch.Tensor:
        """Writes the mean loss's gradient into g (a flat vector like x) and returns the loss."""
        tokens, target = batch[:, :-1], batch[:, 1:].reshape(-1)
        dE, dM, db, *rest = g.split(self.sizes)
        e = self.table.lookup(tokens, self.E)
        first, kept = self.draws, []
        self.draws += len(self.blocks)
        for k, (w, b, A, a, O) in enumerate(self.blocks):
            y, stats = self.norm.forward(e, w, b)
            z, v = torch.addmm(a, y.view(-1, self.dim), A).view(*tokens.shape, 2 * self.dim).split(self.dim, 2)
            h, _ = self.scan.forward(z, v)
            kept.append((e, y, stats, z, v, h))
            e = self.drop((h.view(-1, self.dim) @ O).view(e.shape), first + k, residual=e)
        e = e.view(-1, self.dim)
        h = torch.addmm(self.bias, e, self.M)
        log_p = torch.log_softmax(h @ self.E.t(), 1)
        loss = -log_p.gather(1, target[:, None]).mean()
        d = log_p.exp_()
        d[torch.arange(d.shape[0], device=d.device), target] -= 1.0
        d /= d.shape[0]
        torch.mm(d.t(), h, out=dE.view(self.vocab, self.dim))
        dh = d @ self.E
        torch.mm(e.t(), dh, out=dM.view(self.dim, self.dim))
        db.copy_(dh.sum(0))
        de = (dh @ self.M.t()).view(*tokens.shape, self.dim)
        for k in reversed(range(len(kept))):
            (w, _, A, _, O), (dw, dc, dA, da, dO), (e, y, stats, z, v, h) = self.blocks[k], self._blocks(rest)[k], kept[k]
            do = self.drop.grad(de, first + k).view(-1, self.dim)
            torch.mm(h.view(-1, self.dim).t(), do, out=dO)
            dzv = torch.empty(*tokens.shape, 2 * self.dim, device=e.device)
            dz, dv = dzv.split(self.dim, 2)
            self.scan.grad((do @ O.t()).view(e.shape), z, v, h, dz=dz, dv=dv)
            dzv = dzv.view(-1, 2 * self.dim)
            torch.mm(y.view(-1, self.dim).t(), dzv, out=dA)
            da.copy_(dzv.sum(0))
            de, _, _ = self.norm.grad((dzv @ A.t()).view(e.shape), e, stats, w, add=de, dw=dw, db=dc)
        self.table.grad(tokens, de, out=dE.view(self.vocab, self.dim), accumulate=True)
        return loss


def train(optimizer: str = "adamw", vocab: int = 512, dim: int = 64, sequences: int = 16, length: int = 32, workers: int = 4,
          steps: int = 200, lr: float = 1e-2, max_norm: float = 1.0, seed: int = 0, log=None, blocks: int = 0,
          dropout: float = 0.0) -> list[float]:
    """Trains and returns the loss of every step (mean over the workers).  optimizer: adamw, adamw8 or round.  blocks: of the
    gated recurrence; dropout: in them."""
    device = torch.device("cuda", torch.cuda.current_device())
    corpus, model = Corpus(vocab, seed, device), Bigram(vocab, dim, sequences * length, device, seed, blocks, dropout)
    d, losses = model.x.numel(), []
    grads = [torch.empty(d, device=device) for _ in range(workers)]
    norm, clip = ea.GradNorm([d]), torch.empty(2, device=device)
    if optimizer == "round":
        cfg = ea.EAConfig(d=d, n=workers, qw=W.uniform_q(4, 4096, True), qs=W.uniform_q(8, 4096), alpha=lr, adam_form=1, seed=seed)
        rnd, zero = ea.EARound(cfg), torch.zeros((), device=device)
    else:
        # biases and the norms' weights are vectors: no decay
        opt = ea.AdamW(list(model.x.split(model.sizes)), state_bits=8 if optimizer == "adamw8" else 32,
                       weight_decay=[0.01, 0.01, 0.0] + [0.0, 0.0, 0.01, 0.0, 0.01] * blocks, seed=seed)
        mean = torch.empty(d, device=device)
        pieces = ea.TensorList(mean.split(model.sizes))
    for t in range(steps):
        step_losses = [model.gradient(corpus.batch(sequences, length, 1 + t * workers + i), grads[i]) for i in range(workers)]
        if optimizer == "round":
            for g in grads:  # a factor of NaN in the workers' moments and residuals would stay there
                factor = norm([g], max_norm=max_norm, out=clip)[1]
                torch.where(factor.isnan(), zero, g * factor, out=g)
            rnd.step(grads, model.x)
        else:
            torch.mean(torch.stack(grads), 0, out=mean)
            opt.step(pieces, lr=lr, clip=norm([mean], max_norm=max_norm, out=clip))
        losses.append(torch.stack(step_losses).mean())
        if log and (t % 20 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {float(losses[-1]):.4f}")
    model.table.sync()
    if blocks:
        model.scan.sync()
    if optimizer == "round":
        rnd.sync()
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--optimizer", choices=("adamw", "adamw8", "round"), default="adamw")
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--blocks", type=int, default=0)
    ap.add_argument("--dropout", type=float, default=0.0)
    a = ap.parse_args()
    if a.dropout and not a.blocks:
        ap.error("--dropout is in the blocks: it needs --blocks")
    train(a.optimizer, workers=a.workers, steps=a.steps, lr=a.lr, log=print, blocks=a.blocks, dropout=a.dropout)
