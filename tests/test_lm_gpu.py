"""The operators of include/ea_lm.h on the GPU against plain implementations in 64 bits.

Tolerances come from the operators' own roundings: u = 2^-24 for each operation in binary32, half a unit in the
last place for the rounding to a 16-bit type, and gamma_n = n u / (1 - n u) for a sum of n terms in any order
(Higham, Accuracy and Stability of Numerical Algorithms, Section 4.2), relative to the sum of magnitudes."""
import numpy as np
import pytest
import torch

import paper_2205_14473_gb300 as ea

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}     # relative, of normal values
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}      # spacing of subnormal values


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(*shape, seed=0, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * std).to(dtype)


def _inside(got, want, bound, what=""):
    got, want, bound = (np.asarray(x, dtype=np.float64) for x in (got, want, bound))
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, first at {np.argwhere(bad)[0]}: " \
                          f"{got[bad][0]!r} for {want[bad][0]!r} +- {bound[bad][0]!r}"


def _np(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------ lookup

def _tokens(shape, vocab, seed, dtype=torch.int64, skew=0.0):
    u = torch.rand(shape, generator=_gen(seed), device="cuda", dtype=torch.float64)
    return (u ** (1 + 4 * skew) * vocab).long().clamp_(max=vocab - 1).to(dtype)


def _check_lookup(y, ids, w, scale):
    want = _np(w)[ids.cpu().numpy()] * np.float64(np.float32(scale))
    _inside(_np(y), want, np.abs(want) * (U + HALF_ULP[y.dtype] * (1 + U)) + TINY[y.dtype], "lookup")


@pytest.mark.parametrize("shape", [(1,), (0,), (3, 0), (7,), (2, 33), (1, 257), (4, 3, 5), ()])
@pytest.mark.parametrize("dim", [1, 3, 8, 64, 769, 1600])
def test_lookup_shapes(shape, dim):
    w, ids = _randn(50, dim, seed=1), _tokens(shape, 50, 2)
    table = ea.Embedding(50, dim, max_tokens=512, scale=dim ** 0.5)
    y = table.lookup(ids, w)
    assert y.shape == (*shape, dim)
    _check_lookup(y, ids, w, dim ** 0.5)
    table.sync()


@pytest.mark.parametrize("wt", [F32, BF16, F16])
@pytest.mark.parametrize("yt", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [40, 37])
def test_lookup_types(wt, yt, dim):
    w, ids = _randn(1000, dim, seed=3, dtype=wt), _tokens((300,), 1000, 4, torch.int32)
    _check_lookup(ea.Embedding(1000, dim, 300, scale=0.3).lookup(ids, w, dtype=yt), ids, w, 0.3)


def test_lookup_of_strided_tokens_tables_and_rows():
    """The inputs of next-token training (all but the last of every sequence), a table that is part of a wider
    one, an output that is part of a longer one, and addresses that are aligned to nothing but their element."""
    vocab, dim, b, s = 61, 24, 5, 9
    batch = _tokens((b, s + 1), vocab, 5)
    wide = _randn(vocab, dim + 7, seed=6)
    for off in (0, 1, 3):
        table, y = ea.Embedding(vocab, dim, b * (s + 1)), torch.full((b, s + 2, dim), 7.0, device="cuda")
        table.lookup(batch[:, :-1], wide[:, off:off + dim], out=y[:, 1:-1])
        _check_lookup(y[:, 1:-1], batch[:, :-1], wide[:, off:off + dim], 1.0)
        assert (y[:, 0] == 7).all() and (y[:, -1] == 7).all()
    ids = batch.t()                                     # other orders of the batch
    _check_lookup(table.lookup(ids, wide[:, 2:2 + dim]), ids, wide[:, 2:2 + dim], 1.0)
    ids = batch[:1].expand(4, -1)
    _check_lookup(table.lookup(ids, wide[:, 2:2 + dim]), ids, wide[:, 2:2 + dim], 1.0)
    flat = torch.zeros(vocab * dim + 1, device="cuda", dtype=BF16)
    flat[1:] = _randn(vocab * dim, seed=7, dtype=BF16)
    _check_lookup(table.lookup(batch[:, 2], flat[1:].view(vocab, dim)), batch[:, 2], flat[1:].view(vocab, dim), 1.0)


@pytest.mark.parametrize("dim", [5000, 5003, 2056])
@pytest.mark.parametrize("n", [1, 5, 3000])
def test_lookup_of_long_rows(dim, n):
    """Rows of several pieces, more of them than run at a time."""
    w, ids = _randn(300, dim, seed=dim), _tokens((n,), 300, n)
    _check_lookup(ea.Embedding(300, dim, n, scale=0.5).lookup(ids, w, dtype=BF16), ids, w, 0.5)


@pytest.mark.parametrize("dim", [7, 64, 100])
def test_lookup_of_many_short_rows(dim):
    w, ids = _randn(5000, dim, seed=dim, dtype=BF16), _tokens((300, 1001), 5000, dim)
    _check_lookup(ea.Embedding(5000, dim, 300 * 1001).lookup(ids[:, :-1], w), ids[:, :-1], w, 1.0)


def test_lookup_keeps_infinities_and_nan():
    w = _randn(4, 16, seed=8)
    w[0, 3], w[1, 5], w[2, 7] = float("inf"), float("-inf"), float("nan")
    ids = torch.tensor([3, 2, 1, 0, 2], device="cuda")
    y = ea.Embedding(4, 16, 5, scale=2.0).lookup(ids, w, dtype=BF16)
    assert torch.equal(y.isnan(), w[ids].isnan()) and torch.equal(y.isinf(), w[ids].isinf())
    assert (y.float().isinf() == (w[ids].isinf())).all() and torch.equal(torch.sign(y.float()).nan_to_num(9), torch.sign(w[ids]).nan_to_num(9))


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_tokens_outside_the_table(dtype):
    """A row of zeros, no gradient, and sync() tells; the handle goes on working."""
    vocab, dim = 10, 20
    w, dy = _randn(vocab, dim, seed=9), _randn(6, dim, seed=10)
    ids = torch.tensor([1, -1, 10, 3, 2 ** 31 - 1, 1], device="cuda", dtype=dtype)
    if dtype == torch.int64:
        ids[2] = 2 ** 32 + 1                            # not row 1
    table = ea.Embedding(vocab, dim, 6)
    y = table.lookup(ids, w)
    assert torch.equal(y[[0, 3, 5]], w[[1, 3, 1]]) and (y[[1, 2, 4]] == 0).all()
    with pytest.raises(ea.EAError) as ex:
        table.sync()
    assert ex.value.status == ea.EA_E_DEVICE_CHECK
    table.sync()
    g = table.grad(ids, dy)
    want = torch.zeros(vocab, dim, device="cuda")
    want[1], want[3] = dy[0] + dy[5], dy[3]
    assert torch.equal(g, want)
    with pytest.raises(ea.EAError):
        table.sync()
    table.lookup(ids[:1], w)
    table.sync()


# ------------------------------------------------------------------------------------ table gradient

def _check_grad(got, ids, dy, scale, padding=None, before=None):
    """scale * (sum of count terms, in 32 bits), that rounded, then added and rounded in the table's type."""
    flat, rows = ids.reshape(-1).cpu().numpy().astype(np.int64), _np(dy).reshape(-1, dy.shape[-1])
    keep = np.ones(flat.shape, bool) if padding is None else flat != padding
    want, size = np.zeros(got.shape), np.zeros(got.shape)
    np.add.at(want, flat[keep], rows[keep])
    np.add.at(size, flat[keep], np.abs(rows[keep]))
    count = np.bincount(flat[keep], minlength=got.shape[0])[:, None]
    s = np.float64(np.float32(scale))
    gamma = (count + 1) * U / (1 - (count + 1) * U)
    want, bound = want * s, size * abs(s) * gamma + 2.0 ** -149
    if before is not None:
        want = want + _np(before)
        bound = np.where(count > 0, bound + (np.abs(want) + bound) * U, 0.0)
    store = (np.abs(want) + bound) * HALF_ULP[got.dtype] + TINY[got.dtype]
    _inside(_np(got), want, np.where((count > 0) | (before is None), bound + store, 0.0), "gradient")


# token counts around the sizes at which work is split, and tables of one, two and three radix digits
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 1023, 1025, 4097, 20_000])
@pytest.mark.parametrize("vocab,skew", [(1, 0.0), (5, 0.0), (300, 1.0), (70_000, 1.0)])
def test_grad_sizes(n, vocab, skew):
    dim = 24
    ids, dy = _tokens((n,), vocab, n + vocab, skew=skew), _randn(n, dim, seed=n)
    table = ea.Embedding(vocab, dim, n, scale=1.5)
    got = table.grad(ids, dy)
    _check_grad(got, ids, dy, 1.5)
    assert torch.equal(got, table.grad(ids, dy, out=torch.full_like(got, float("nan"))))
    table.sync()


@pytest.mark.parametrize("dim", [1, 2, 3, 5, 8, 17, 100, 256, 769, 1600, 2056])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grad_widths(dim, dtype):
    n, vocab = 700, 90
    ids, dy = _tokens((n,), vocab, dim, skew=0.5), _randn(n, dim, seed=dim, dtype=dtype)
    _check_grad(ea.Embedding(vocab, dim, n).grad(ids, dy), ids, dy, 1.0)


@pytest.mark.parametrize("yt", [F32, BF16, F16])
@pytest.mark.parametrize("wt", [F32, BF16, F16])
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("dim", [64, 33])
def test_grad_types(yt, wt, tied, dim):
    n, vocab = 500, 200
    ids, dy = _tokens((n,), vocab, 11, torch.int32, skew=1.0), _randn(n, dim, seed=12, dtype=yt)
    before = _randn(vocab, dim, seed=13, dtype=wt)
    out = before.clone()
    got = ea.Embedding(vocab, dim, n, scale=8.0).grad(ids, dy, out=out, accumulate=tied)
    assert got is out
    _check_grad(got, ids, dy, 8.0, before=before if tied else None)


@pytest.mark.parametrize("n", [3000, 150_000])
@pytest.mark.parametrize("tied", [False, True])
def test_grad_of_one_token_and_of_padding(n, tied):
    """Every token the same (one sum over all rows); every other one padding; nothing but padding."""
    vocab, dim = 40, 16
    dy, before = _randn(n, dim, seed=14), _randn(vocab, dim, seed=15)
    table = ea.Embedding(vocab, dim, n, padding_idx=0)
    for ids in (torch.full((n,), 39, device="cuda"), torch.arange(n, device="cuda") % 2 * 7,
                torch.zeros(n, device="cuda", dtype=torch.int64)):
        got = table.grad(ids, dy, out=before.clone(), accumulate=tied)
        _check_grad(got, ids, dy, 1.0, padding=0, before=before if tied else None)


@pytest.mark.parametrize("n,vocab,dim", [(70_000, 50_257, 40), (200_000, 1000, 40), (131_073, 3, 40), (70_000, 200_000, 9),
                                         (65_536, 300, 8), (65_537, 131_073, 8)])
def test_grad_of_many_tokens(n, vocab, dim):
    ids, dy = _tokens((n,), vocab, 16, skew=1.0), _randn(n, dim, seed=17, dtype=BF16)
    table = ea.Embedding(vocab, dim, n)
    got = table.grad(ids, dy)
    _check_grad(got, ids, dy, 1.0)
    for _ in range(3):
        assert torch.equal(table.grad(ids, dy), got)


@pytest.mark.parametrize("n,vocab,dim", [(20_000, 300, 64), (3000, 7, 1600), (70_000, 1000, 104), (5000, 40, 8)])
@pytest.mark.parametrize("yt,wt", [(BF16, F32), (F32, F32), (F32, BF16), (F16, F16)])
@pytest.mark.parametrize("tied", [False, True])
def test_grad_has_the_same_bits_at_any_alignment(n, vocab, dim, yt, wt, tied):
    """The order of the sums goes by the tokens and the sizes: rows and tables off a 16-byte boundary, and rows with gaps
    between them, get the bits of aligned ones (runs of one token that cross many pieces of the sorted list)."""
    ids, dy, before = _tokens((n,), vocab, 30, skew=0.5), _randn(n, dim, seed=31, dtype=yt), _randn(vocab, dim, seed=32, dtype=wt)
    table = ea.Embedding(vocab, dim, n, scale=1.5)
    want = table.grad(ids, dy, out=before.clone(), accumulate=tied)

    def off(t, k):
        flat = torch.empty(t.numel() + k, device="cuda", dtype=t.dtype)
        flat[k:] = t.flatten()
        return flat[k:].view(t.shape)

    wide = torch.empty(n, dim + 3, device="cuda", dtype=yt)
    wide[:, 1:dim + 1] = dy
    for rows, out in ((dy, off(before, 1)), (off(dy, 1), before.clone()), (off(dy, 3), off(before, 5)), (wide[:, 1:dim + 1], before.clone())):
        assert torch.equal(table.grad(ids, rows, out=out, accumulate=tied), want)
    by_batch = table.grad(ids.view(-1, 4).to(torch.int32), dy.view(-1, 4, dim), out=before.clone(), accumulate=tied)
    assert torch.equal(by_batch, want)


def test_grad_of_strided_inputs():
    vocab, dim, b, s = 30, 12, 6, 50
    batch, dh = _tokens((b, s + 1), vocab, 18), _randn(b, s + 1, dim + 4, seed=19)
    table = ea.Embedding(vocab, dim, b * (s + 1))
    for dy in (dh[:, :-1, :dim], dh[:, 1:, 1:dim + 1], dh[:, :1, :dim].expand(b, s, dim), dh[:, :-1, :2 * dim:2][..., :1].expand(b, s, dim)):
        _check_grad(table.grad(batch[:, :-1], dy), batch[:, :-1], dy, 1.0)
    flat = torch.full((vocab * dim + 3,), 5.0, device="cuda")    # a piece of a flat gradient, at any offset
    for off in (0, 1, 3):
        flat.fill_(5.0)
        out = flat[off:off + vocab * dim].view(vocab, dim)
        table.grad(batch, dh[..., :dim], out=out)
        _check_grad(out, batch, dh[..., :dim], 1.0)
        assert (flat[:off] == 5).all() and (flat[off + vocab * dim:] == 5).all()
    wide = torch.full((vocab, dim + 5), 5.0, device="cuda")
    table.grad(batch, dh[..., :dim], out=wide[:, 2:2 + dim])
    _check_grad(wide[:, 2:2 + dim], batch, dh[..., :dim], 1.0)
    assert (wide[:, :2] == 5).all() and (wide[:, 2 + dim:] == 5).all()


@pytest.mark.parametrize("shape", [(0,), (4, 0)])
def test_grad_of_no_tokens(shape):
    ids, dy = torch.zeros(shape, device="cuda", dtype=torch.int64), torch.zeros(*shape, 8, device="cuda")
    table, out = ea.Embedding(20, 8, 4), torch.full((20, 8), 3.0, device="cuda")
    assert (table.grad(ids, dy, out=out, accumulate=True) == 3).all()
    assert (table.grad(ids, dy, out=out) == 0).all()


def test_infinities_stay_in_their_rows():
    ids, dy = torch.tensor([4, 1, 4, 2], device="cuda"), _randn(4, 8, seed=20)
    dy[0, 2], dy[3, 5] = float("inf"), float("nan")
    g = ea.Embedding(6, 8, 4).grad(ids, dy)
    assert g[4, 2] == float("inf") and g[2, 5].isnan() and int((~g.isfinite()).sum()) == 2


def test_gradient_against_differences():
    """<grad, E> for E one at (v, j) against the change of sum(c * lookup) when w[v, j] moves by h: the loss is
    linear in w, so the difference quotient is exact but for the roundings of y (2 u |y| a term and side)."""
    vocab, dim, n, h = 7, 6, 50, 0.5
    w, c, ids = _randn(vocab, dim, seed=21), _randn(n, dim, seed=22), _tokens((n,), vocab, 23)
    table = ea.Embedding(vocab, dim, n, scale=1.25)
    g = _np(table.grad(ids, c))
    for v in range(vocab):
        for j in range(dim):
            side = []
            for sign in (1, -1):
                x = w.clone()
                x[v, j] += sign * h
                side.append(((_np(c) * _np(table.lookup(ids, x))).sum(), float(x[v, j])))
            quotient = (side[0][0] - side[1][0]) / (side[0][1] - side[1][1])
            terms = np.abs(_np(c)[ids.cpu().numpy() == v, j]).sum() * 1.25
            bound = terms * (2 * U * (abs(float(w[v, j])) + h) / h + (n + 1) * 2 * U) + 1e-12
            assert abs(quotient - g[v, j]) <= bound


# ------------------------------------------------------------------------------------------- norm

def _check_norm(out, parts, max_norm=np.inf, grad_scale=1.0):
    norm = abs(grad_scale) * np.sqrt(sum(float((_np(p) ** 2).sum()) for p in parts))
    factor = grad_scale * min(1.0, max_norm / norm) if norm > 0 else grad_scale
    # at most 32 squares are summed in 32 bits, the rest in 64, and a square root halves a relative error
    rel = 0.5 * 33 * U + 2 * U
    _inside(_np(out), [norm, factor], [norm * rel + 2.0 ** -149, abs(factor) * rel], "norm")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [31, 32, 33], [1023, 1024, 1025, 4097], [1_000_003], [5, 70_001, 0, 3, 2_000_000]])
def test_norm_sizes(dtype, sizes):
    flat = _randn(sum(sizes), seed=len(sizes), dtype=dtype)
    parts = list(flat.split(sizes))                        # pieces at any alignment
    norm = ea.GradNorm(sizes, dtype)
    out = norm(parts, max_norm=0.5)
    _check_norm(out, parts, 0.5)
    assert torch.equal(out, norm(ea.TensorList(parts), max_norm=0.5))
    _check_norm(norm(parts, max_norm=1e9, grad_scale=-0.25), parts, 1e9, -0.25)


def test_norm_of_many_tensors():
    sizes = [(i * 7919) % 1500 for i in range(2000)]       # several launches
    parts = list(_randn(sum(sizes), seed=24).split(sizes))
    norm = ea.GradNorm(sizes)
    _check_norm(norm(parts, max_norm=2.0), parts, 2.0)
    _check_norm(norm(parts, max_norm=3.0), parts, 3.0)


@pytest.mark.parametrize("mag", [1e-44, 1e-38, 1e-30, 1e-20, 1e-12, 1.0, 1e12, 1e18, 1e20, 1e30, 1e34])
def test_norm_of_any_magnitude(mag):
    """Squares that leave binary32's range at either end, alone and beside ordinary values."""
    x = (_randn(5000, seed=25) * np.float32(mag)).clamp(-3e38, 3e38)
    _check_norm(ea.GradNorm([5000])([x], max_norm=1.0), [x], 1.0)
    y = torch.cat([x, _randn(5000, seed=26)])
    _check_norm(ea.GradNorm([10_000])([y]), [y])
    z = torch.cat([torch.zeros(4000, device="cuda"), x[:1], torch.zeros(999, device="cuda")])
    _check_norm(ea.GradNorm([5000])([z], max_norm=1.0), [z], 1.0)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_norm_of_what_is_not_finite(bad, dtype):
    x = _randn(3000, seed=27, dtype=dtype)
    x[1234] = bad
    out = ea.GradNorm([3000], dtype)([x], max_norm=1.0)
    assert not bool(out[0].isfinite()) and bool(out[1].isnan())
    big = torch.full((100,), 3e38, device="cuda")          # finite values, a norm beyond binary32
    out = ea.GradNorm([100])([big], max_norm=1.0)
    assert bool(out[0].isinf()) and bool(out[1].isnan())


def test_norm_of_nothing():
    out = ea.GradNorm([10])([torch.zeros(10, device="cuda")], max_norm=0.0, grad_scale=2.0)
    assert out.tolist() == [0.0, 2.0]
    assert ea.GradNorm([0])([torch.zeros(0, device="cuda")], max_norm=1.0).tolist() == [0.0, 1.0]


# ------------------------------------------------------------------------------------------ AdamW

B1, B2 = np.float64(np.float32(0.9)), np.float64(np.float32(0.999))


def _adamw_bound(p, g, m, v, lr, decay, t, eps, ptype):
    """One step in 64 bits from these (float64) values, and how far the step's roundings may take each result."""
    root, bc1 = np.sqrt(1 - B2 ** t), 1 - B1 ** t
    m1, v1 = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    am = np.abs(B1 * m) + np.abs((1 - B1) * g)
    em, ev = am * 4 * U + 2.0 ** -147, v1 * 5 * U + 2.0 ** -147      # g's product, two products, a sum
    den = np.sqrt(v1) + eps * root
    eden = np.sqrt(v1 + ev) - np.sqrt(v1) + 4 * U * den               # root, its rounding, epsilon's, the sum's
    a = lr * root / bc1
    step = a * m1 / den
    estep = a * (am + em) / den * (8 * U + eden / den) + a * em / den + 2.0 ** -147
    new = p - (lr * decay * p + step)
    enew = estep + (np.abs(lr * decay * p) * 4 + np.abs(new)) * U
    return (new, enew + (np.abs(new) + enew) * HALF_ULP[ptype] + TINY[ptype]), (m1, em), (v1, ev)


@pytest.mark.parametrize("ptype,gtype,copy", [(F32, F32, None), (F32, BF16, BF16), (F32, F16, F16), (BF16, BF16, None),
                                              (BF16, F32, None), (BF16, F16, None), (F32, F32, BF16)])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 255, 256, 257], [64, 9408, 1000, 513], [40_001]])
def test_adamw_32(ptype, gtype, copy, sizes):
    n = sum(sizes)
    p, clip = _randn(n, seed=30, dtype=ptype), torch.tensor([5.0, 0.3], device="cuda")
    decay = [0.1 if k > 100 else 0.0 for k in sizes]
    scale = [1.0 + 0.5 * (i % 2) for i in range(len(sizes))]
    copies = None if copy is None else torch.zeros(n, device="cuda", dtype=copy)
    opt = ea.AdamW(list(p.split(sizes)), weight_decay=decay, lr_scale=scale, grad_dtype=gtype, eps=1e-6,
                   copies=None if copy is None else list(copies.split(sizes)))
    lr, eps = np.float64(np.float32(1e-2)), np.float64(np.float32(1e-6))
    d, s = np.repeat(np.float32(decay).astype(float), sizes), np.repeat(np.float32(scale).astype(float), sizes)
    factor = float(clip[1])
    for t in range(1, 4):
        g = _randn(n, seed=30 + t, dtype=gtype, std=10.0 ** (t - 2))
        before = _np(p), _np(torch.cat(opt.states["m"])), _np(torch.cat(opt.states["v"]))
        opt.step(list(g.split(sizes)), lr=1e-2, clip=clip if t != 2 else None)
        new, m, v = _adamw_bound(before[0], _np(g) * (factor if t != 2 else 1.0), *before[1:], lr * s, d, t, eps, ptype)
        _inside(_np(torch.cat(opt.states["m"])), *m, "m")
        _inside(_np(torch.cat(opt.states["v"])), *v, "v")
        _inside(_np(p), *new, "p")
        if copy is not None:
            _inside(_np(copies), new[0], new[1] + (np.abs(new[0]) + new[1]) * HALF_ULP[copy] + TINY[copy], "copy")
        assert opt.t == t


def _philox(seed, counter):
    """Philox4x32-10 of the C oracle's words, in numpy."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        k0, k1 = ((k[0] + r * 0x9E3779B9) & 0xFFFFFFFF), ((k[1] + r * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & np.uint64(0xFFFFFFFF),
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & np.uint64(0xFFFFFFFF)]
    return np.stack(c)


def test_philox_of_this_file():
    """The published known-answer vectors of the generator."""
    assert [int(x) for x in _philox(0, [0, 0, 0, 0])] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert [int(x) for x in _philox((ones << 32) | ones, [ones] * 4)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def _check_codes(q, scale, x, ex, random, keep_nonzero, what):
    """q (values of the codes) and scale (of every block) against x (64 bits, known to ex): the scale is the
    smallest power of two that brings the largest magnitude to 448, and a code is the grid point that the random
    number takes |x| / scale to, unless that lies within ex of the next one's threshold."""
    n = x.size
    for b in range(-(-n // 256)):
        s = slice(256 * b, min(n, 256 * b + 256))
        top, off = np.abs(x[s]).max(), ex[s][np.abs(x[s]).argmax()]
        want = [2.0 ** max(-126, int(np.ceil(np.log2(v / 448)))) if v > 0 else 2.0 ** -126 for v in (max(top - off, 0), top + off)]
        assert want[0] <= scale[b] <= want[1], (what, b, scale[b], want)
        y, e = np.abs(x[s]) / scale[b], ex[s] / scale[b]
        grid = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
        ends = [np.maximum(y + sign * e, 0) * (x[s] != 0) for sign in (-1, 1)]
        lo, hi = (np.floor(end / grid + random[s] / 65536.0) * grid for end in ends)
        if keep_nonzero:
            lo, hi = (np.where(end > 0, np.maximum(v, 2.0 ** -9), v) for end, v in zip(ends, (lo, hi)))
        got = np.abs(q[s])
        bad = (got < lo) | (got > hi) | (got.astype(np.float32) != got)
        assert not bad.any(), (what, b, np.argwhere(bad)[:3], got[bad][:3], lo[bad][:3], y[bad][:3])
        assert (np.sign(q[s])[got > 0] == np.sign(x[s])[got > 0]).all()
        assert (lo != hi).mean() < 0.02                     # the threshold's neighbourhood is all that is left open


@pytest.mark.parametrize("ptype,gtype,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None), (BF16, F16, None)])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 255, 256, 257], [64, 9408, 1000, 513], [20_001], [2048, 512]])
def test_adamw_8(ptype, gtype, copy, sizes):
    n, seed = sum(sizes), 0x123456789ABCDEF
    p, clip = _randn(n, seed=40, dtype=ptype), torch.tensor([5.0, 0.3], device="cuda")
    copies = None if copy is None else torch.zeros(n, device="cuda", dtype=copy)
    opt = ea.AdamW(list(p.split(sizes)), state_bits=8, weight_decay=0.1, grad_dtype=gtype, seed=seed,
                   copies=None if copy is None else list(copies.split(sizes)))
    lr, eps, decay = (np.float64(np.float32(x)) for x in (1e-2, 1e-8, 0.1))
    for t in range(1, 5):
        g = _randn(n, seed=40 + t, dtype=gtype) * torch.rand(n, generator=_gen(t), device="cuda").pow_(8).to(gtype)
        g[::7] = 0
        parts, before = list(g.split(sizes)), []
        for i in range(len(sizes)):
            rep = lambda k: np.repeat(_np(opt.states[k][i]), 256)[:sizes[i]]  # noqa: E731
            before.append((_np(opt.params.tensors[i]), _np(opt.states["m"][i]) * rep("m_scale"),
                           (_np(opt.states["r"][i]) * rep("r_scale")) ** 2))
        opt.step(parts, lr=1e-2, clip=clip)
        for i, size in enumerate(sizes):
            if size == 0:
                continue
            p0, m0, v0 = before[i]
            new, m, v = _adamw_bound(p0, _np(parts[i]) * float(clip[1]), m0, v0 , lr, decay, t, eps, ptype)
            v = (v[0], v[1] + v0 * U)                        # the root's square is rounded once more
            enew = new[1] + np.abs(new[0] - p0) * 2 * U
            _inside(_np(opt.params.tensors[i]), new[0], enew, "p")
            if copy is not None:
                c = _np(opt.copies[i])
                _inside(c, new[0], enew + (np.abs(new[0]) + enew) * HALF_ULP[copy] + TINY[copy], "copy")
            j = np.arange(size)
            words = np.take_along_axis(_philox(seed, [j // 4 & 0xFFFFFFFF, j // 4 >> 32, np.full(size, i), np.full(size, t - 1)]),
                                       (j % 4)[None], 0)[0].astype(np.int64)
            _check_codes(_np(opt.states["m"][i]), _np(opt.states["m_scale"][i]), *m, words & 0xFFFF, False, f"m of {i}")
            r = np.sqrt(v[0])
            _check_codes(_np(opt.states["r"][i]), _np(opt.states["r_scale"][i]), r, np.sqrt(v[0] + v[1]) - r + 2 * U * r,
                         words >> 16, True, f"r of {i}")


@pytest.mark.parametrize("ptype,gtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F16), (BF16, F32), (F32, F16)])
@pytest.mark.parametrize("mag", [1e-3, 1e-19, 1e13])
def test_adamw_8_states_are_binary32(ptype, gtype, mag):
    """The moments and the root before they are rounded to 8 bits, one binary32 rounding per operation: torch's
    elementary operations, each its own kernel, and the format's rounding in integers give the same bytes."""
    if mag > 1e4 and gtype == F16:
        mag = 1e4                                           # the type's range; 1e13 has squares beyond 2^60
    n = 3_000_000 if mag == 1e-3 else 300_000
    p, opt = _randn(n, seed=90, dtype=ptype), None
    factor = torch.tensor([1.0, 0.37], device="cuda")
    opt = ea.AdamW([p], state_bits=8, grad_dtype=gtype, seed=77)
    blk = torch.arange(n, device="cuda") // 256
    j = np.arange(n // 4)
    for t in range(3):
        g = (_randn(n, seed=91 + t) * torch.rand(n, generator=_gen(t), device="cuda").pow_(4) * mag).to(gtype)
        old = {k: v[0].float().clone() for k, v in opt.states.items()}
        opt.step([g], lr=1e-3, clip=factor)
        gf = g.float() * factor[1]
        m = old["m"] * old["m_scale"][blk] * 0.9 + gf * float(np.float32(1) - np.float32(0.9))
        r = old["r"] * old["r_scale"][blk]
        root = (r * r * 0.999 + gf * gf * float(np.float32(1) - np.float32(0.999))).sqrt()
        words = torch.from_numpy(_philox(77, [j, j * 0, j * 0, j * 0 + t]).T.reshape(-1).astype(np.int64)).cuda()
        for k, x, r16 in (("m", m, words & 0xFFFF), ("r", root, words >> 16)):
            top = torch.zeros(-(-n // 256), device="cuda").scatter_reduce_(0, blk, x.abs(), "amax")
            e = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 135).clamp(min=-126)
            y = x.abs() * ((127 - e) << 23).view(torch.float32)[blk]
            q = ((y.view(torch.int32) + (r16 << 4).to(torch.int32)) & -0x100000).view(torch.float32)
            q = torch.where(y >= 2.0 ** -6, q, torch.floor(y * 512 + r16.float() * 2.0 ** -16) * 2.0 ** -9)
            q = torch.where(root > 0, q.clamp(min=2.0 ** -9), q) if k == "r" else torch.copysign(q, x)
            assert torch.equal(opt.states[k + "_scale"][0], ((127 + e) << 23).view(torch.float32)), (k, t)
            got = opt.states[k][0].float()
            assert torch.equal(got, q), (k, t, int((got != q).sum()))


def test_adamw_8_square_root():
    """The 8-bit step's square root is the correctly rounded one for every value that it is taken of: a root of a block's
    maximum that came out one unit too large would have no code."""
    import ctypes

    unequal = ctypes.c_uint64(1)
    assert ea.lib().ea_adamw_selftest_sqrt(torch.cuda.current_stream().cuda_stream, ctypes.byref(unequal)) == ea.EA_OK
    assert unequal.value == 0


def test_adamw_8_rounding_is_unbiased():
    """The mean of the held first moment over many coordinates with the same value: within 6 standard deviations
    of that value (a deviation is at most half the grid's spacing)."""
    n = 1 << 20
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.7, device="cuda")
    opt = ea.AdamW([p], state_bits=8, seed=5, weight_decay=0.0)
    opt.step([g], lr=0.0)
    m = _np(opt.states["m"][0]) * _np(opt.states["m_scale"][0])[0]
    x = (1 - B1) * 0.7
    assert len(np.unique(m)) == 2
    assert abs(m.mean() - x) <= 6 * 0.5 * np.ptp(m) / np.sqrt(n) + x * 4 * U
    assert (p == 0).all()


def test_adamw_8_holds_what_is_not_finite_as_nan():
    """One infinite and one NaN gradient: their coordinates only, and the block's scale from the others."""
    p, g = _randn(600, seed=50), _randn(600, seed=51)
    a, b = [x.clone() for x in (p, p)], g.clone()
    b[5], b[300] = float("inf"), float("nan")
    one, two = (ea.AdamW([x], state_bits=8, seed=9) for x in a)
    one.step([g], lr=1e-3)
    two.step([b], lr=1e-3)
    keep = torch.ones(600, dtype=torch.bool, device="cuda")
    keep[[5, 300]] = False
    assert torch.equal(a[0][keep], a[1][keep])
    for k in ("m", "r"):
        x, y = one.states[k][0].float(), two.states[k][0].float()
        assert y[[5, 300]].isnan().all() and y[keep].isfinite().all()
        s = [o.states[k + "_scale"][0].repeat_interleave(256)[:600] for o in (one, two)]
        same = (s[0] == s[1]) & keep                         # a block whose largest was replaced has another scale
        assert torch.equal(x[same], y[same]) and int(same.sum()) > 0


def test_adamw_skips_a_step_whose_factor_is_nan():
    sizes = [300, 5]
    for bits in (32, 8):
        p = _randn(305, seed=52)
        opt = ea.AdamW(list(p.split(sizes)), state_bits=bits)
        norm = ea.GradNorm(sizes)
        g = _randn(305, seed=53)
        opt.step(list(g.split(sizes)), lr=1e-2, clip=norm(list(g.split(sizes)), max_norm=1.0))
        kept = [p.clone()] + [t.clone() for v in opt.states.values() for t in v]
        g[7] = float("inf")
        opt.step(list(g.split(sizes)), lr=1e-2, clip=norm(list(g.split(sizes)), max_norm=1.0))
        now = [p] + [t for v in opt.states.values() for t in v]
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(kept, now))
        assert opt.t == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_many_tensors_and_any_alignment(bits):
    """1,000 tensors (several launches) at every alignment, against the same tensors at addresses of their own:
    the same bits."""
    sizes = [(i * 7919) % 700 for i in range(1000)]
    n = sum(sizes)
    p, g = _randn(n, seed=54), _randn(n, seed=55, dtype=BF16)
    flat, grads = p.clone(), g.clone()
    ps = [t.clone() for t in p.split(sizes)]
    opts = [ea.AdamW(list(flat.split(sizes)), state_bits=bits, grad_dtype=BF16, seed=3), ea.AdamW(ps, state_bits=bits, grad_dtype=BF16, seed=3,
            states={k: [t.clone() for t in v] for k, v in ea.AdamW(ps, state_bits=bits).states.items()})]
    for t in range(3):
        opts[0].step(list(grads.split(sizes)), lr=1e-2)
        opts[1].step([x.clone() for x in grads.split(sizes)], lr=1e-2)
    assert torch.equal(flat, torch.cat(ps))
    for k in opts[0].states:
        x, y = (torch.cat([t.view(torch.uint8) for t in o.states[k]]) for o in opts)
        assert torch.equal(x, y), k
    assert opts[0].t == opts[1].t == 3


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_resumes(bits):
    """Two steps, then a new handle from the states and the count: the bits of three steps."""
    p, q = _randn(5000, seed=56), _randn(5000, seed=56)
    gs = [_randn(5000, seed=57 + t) for t in range(3)]
    opt = ea.AdamW([p], state_bits=bits, seed=4)
    for g in gs:
        opt.step([g], lr=1e-2)
    first = ea.AdamW([q], state_bits=bits, seed=4)
    for g in gs[:2]:
        first.step([g], lr=1e-2)
    ea.AdamW([q], state_bits=bits, seed=4, states=first.states, step=first.t).step([gs[2]], lr=1e-2)
    _inside(_np(q), _np(p), np.abs(_np(p)) * U * 2, "p")     # beta^t is formed as a power here, as a product there
    for k in opt.states:
        assert torch.equal(opt.states[k][0].view(torch.uint8), first.states[k][0].view(torch.uint8))


def test_adamw_agrees_with_torch():
    p = _randn(3000, seed=60)
    q = torch.nn.Parameter(p.clone().double())
    opt, ref = ea.AdamW([p], weight_decay=0.1), torch.optim.AdamW([q], lr=1e-2, weight_decay=0.1, eps=1e-8)
    for t in range(20):
        g = _randn(3000, seed=61 + t)
        opt.step([g], lr=1e-2)
        q.grad = g.double()
        ref.step()
    # twenty steps of at most 1e-2 (1 + 1 / sqrt(1 - beta2)) each, twenty roundings of 8 u apiece
    _inside(_np(p), _np(q.data), np.abs(_np(q.data)) * 20 * 2 * U + 20 * 0.33 * 20 * 10 * U, "p")


# ------------------------------------------------------------------------- offsets beyond 2^31 elements

FAR = 2 ** 31 + 4096


def test_far_rows_of_tables_and_outputs():
    """A table of more than 2^31 elements, and rows that lie as far apart."""
    dim = 1024
    vocab = FAR // dim
    w = torch.empty(vocab, dim, device="cuda", dtype=BF16)
    ids = torch.tensor([[vocab - 1, 0, vocab - 2], [vocab // 2, vocab - 1, 1]], device="cuda")
    rows = _randn(2, 3, dim, seed=100, dtype=BF16)
    w[ids] = rows
    rows = w[ids]
    table, flat = ea.Embedding(vocab, dim, 6), torch.empty(FAR + 3 * dim, device="cuda", dtype=BF16)
    assert torch.equal(table.lookup(ids, w), rows)
    far = flat.as_strided((2, 3, dim), (2 ** 31, dim, 1))
    assert torch.equal(table.lookup(ids, w, out=far), rows)
    narrow, few = ea.Embedding(FAR // 64, 64, 6), ids * 16
    assert torch.equal(narrow.lookup(few, w.view(-1, 64)), w.view(-1, 64)[few])
    # the gradient of that table, from rows that lie far apart
    w.fill_(float("nan"))
    table.grad(ids, far, out=w)
    want = far.reshape(6, dim).clone()
    want[0] = (want[0].float() + want[4].float()).to(BF16)
    got = w[ids].view(6, dim)
    assert torch.equal(got[[0, 1, 2, 3, 5]], want[[0, 1, 2, 3, 5]])
    assert int(torch.count_nonzero(w)) == int(torch.count_nonzero(got[[0, 1, 2, 3, 5]]))


@pytest.mark.parametrize("off", [0, 1])
def test_far_coordinates_of_the_norm(off):
    x = torch.zeros(FAR + off, device="cuda", dtype=BF16)[off:]
    x[:1000], x[-1000:] = _randn(1000, seed=101, dtype=BF16), _randn(1000, seed=102, dtype=BF16)
    _check_norm(ea.GradNorm([FAR], BF16)([x], max_norm=1.0), [torch.cat([x[:1000], x[-1000:]])], 1.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_far_coordinates_of_adamw(bits):
    """The first step moves a coordinate by lr g / (|g| + eps), wherever it lies, and nothing else: with eps far below
    |g|, by lr within the step's roundings (and the parameter's) of either sign."""
    p, g = torch.zeros(FAR, device="cuda", dtype=BF16), torch.zeros(FAR, device="cuda", dtype=BF16)
    for part in (slice(0, 1000), slice(2 ** 31 - 500, 2 ** 31 + 500), slice(FAR - 1000, FAR)):
        g[part] = torch.sign(_randn(1000, seed=103))
    opt = ea.AdamW([p], state_bits=bits, weight_decay=0.1)
    opt.step([g], lr=0.5)
    assert int(torch.count_nonzero(p)) == 3000 and int(torch.count_nonzero(opt.states["m"][0].view(torch.uint8))) >= 3000
    for part in (slice(0, 1000), slice(2 ** 31 - 500, 2 ** 31 + 500), slice(FAR - 1000, FAR)):
        _inside(_np(p[part]), -0.5 * _np(g[part]), 0.5 * (20 * U + 1e-6 + HALF_ULP[BF16]), "p")


# ------------------------------------------------------------------------- streams, graphs, refusals

def test_another_current_stream():
    """Handles of one stream called while others are current: the results of one stream."""
    vocab, dim, n = 1000, 64, 4000
    ids, w, dy = _tokens((n,), vocab, 70), _randn(vocab, dim, seed=71), _randn(n, dim, seed=72)
    p, sizes = _randn(vocab * dim, seed=73), [vocab * dim]

    def run(stream):
        table, norm, q = ea.Embedding(vocab, dim, n), ea.GradNorm(sizes), p.clone()
        opt = ea.AdamW([q], state_bits=8, seed=1)
        torch.cuda.synchronize()
        out = []
        for t in range(5):
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                late = dy * (t + 1)
                y = table.lookup(ids, w)
                g = table.grad(ids, late + y)
                opt.step([g.view(-1)], lr=1e-3, clip=norm([g.view(-1)], max_norm=1.0))
                out += [y.clone(), g.clone(), q.clone()]
        torch.cuda.synchronize()
        return out

    assert all(torch.equal(x, y) for x, y in zip(run(None), run(torch.cuda.Stream())))


def test_written_tensors_count_as_modified():
    """A backward pass that saved what a call then writes to is refused, as after torch's own operations in place."""
    vocab, dim = 10, 8
    w, ids, dy = _randn(vocab, dim, seed=77), torch.tensor([1, 2], device="cuda"), _randn(2, dim, seed=78)
    table, norm = ea.Embedding(vocab, dim, 2), ea.GradNorm([5])
    p, c, g = torch.nn.Parameter(_randn(5, seed=79)), torch.zeros(5, device="cuda", dtype=BF16), _randn(5, seed=80)
    opt = ea.AdamW([p], copies=[c], grad_dtype=F32)
    row, dw, out = torch.empty(2, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda"), torch.empty(2, device="cuda")
    flat = torch.zeros(9, device="cuda")
    pieces = ea.AdamW(list(flat.split([4, 5])), state_bits=8)
    for f, written in ((lambda: opt.step([g], lr=1e-3), (p, c, opt.states["m"][0])),
                       (lambda: pieces.step([g[:4], g], lr=1e-3), (flat, pieces.params.tensors[1])),
                       (lambda: table.lookup(ids, w, out=row), (row,)),
                       (lambda: table.grad(ids, dy, out=dw, accumulate=True), (dw,)), (lambda: norm([g], out=out), (out,))):
        for t in written:
            x = torch.ones_like(t, requires_grad=True)
            loss = (x * t).sum()
            f()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    with torch.inference_mode():                             # tensors that have no count
        dw = torch.zeros(vocab, dim, device="cuda")
        assert torch.equal(table.grad(ids, dy, out=dw), table.grad(ids, dy))
        q = torch.zeros(5, device="cuda")
        ea.AdamW([q]).step([g], lr=1e-3)


def test_a_lookup_has_no_graph():
    w = torch.nn.Parameter(_randn(10, 8, seed=81))
    y = ea.Embedding(10, 8, 2).lookup(torch.tensor([1, 2], device="cuda"), w)
    assert not y.requires_grad and torch.equal(y, w.detach()[[1, 2]])


def test_graph_replays_count_steps():
    vocab, dim, n = 500, 32, 600
    ids, dy, p = _tokens((n,), vocab, 74), _randn(n, dim, seed=75), _randn(vocab * dim, seed=76)

    def make(q):
        return ea.Embedding(vocab, dim, n), ea.GradNorm([vocab * dim]), ea.AdamW([q], state_bits=8, seed=2)

    def step(table, norm, opt, g, clip):
        table.grad(ids, dy, out=g)
        norm([g.view(-1)], max_norm=1.0, out=clip)
        opt.step([g.view(-1)], lr=1e-2, clip=clip)

    q, r = p.clone(), p.clone()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops, g, clip = make(q), torch.empty(vocab, dim, device="cuda"), torch.empty(2, device="cuda")
        step(*ops, g, clip)                                  # modules are loaded before the capture
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(*ops, g, clip)
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    plain, g2, clip2 = make(r), torch.empty(vocab, dim, device="cuda"), torch.empty(2, device="cuda")
    for _ in range(5):
        step(*plain, g2, clip2)
    assert ops[2].t == plain[2].t == 5 and torch.equal(q, r) and torch.equal(g, g2)


def test_refusals():
    vocab, dim = 10, 8
    w, ids = _randn(vocab, dim, seed=80), torch.tensor([1, 2], device="cuda")
    table = ea.Embedding(vocab, dim, 4)
    dy = _randn(2, dim, seed=81)

    def no(status, f, *a, **k):
        with pytest.raises(ea.EAError) as ex:
            f(*a, **k)
        assert ex.value.status == status and str(ex.value)

    no(ea.EA_E_INVAL, table.lookup, torch.zeros(5, dtype=torch.int64, device="cuda"), w)      # more than max_tokens
    no(ea.EA_E_INVAL, table.lookup, ids.float(), w)
    no(ea.EA_E_INVAL, table.lookup, ids.cpu(), w)
    no(ea.EA_E_INVAL, table.lookup, ids, w.cpu())
    no(ea.EA_E_INVAL, table.lookup, ids, w[:9])
    no(ea.EA_E_INVAL, table.lookup, ids, w.double())
    no(ea.EA_E_INVAL, table.lookup, ids, _randn(dim, vocab, seed=1).t())
    no(ea.EA_E_INVAL, table.lookup, ids, w[:1].expand(vocab, dim))
    no(ea.EA_E_INVAL, table.lookup, ids, w, out=torch.empty(3, dim, device="cuda"))
    no(ea.EA_E_INVAL, table.lookup, ids, w, out=torch.empty(2, dim, device="cuda"), dtype=BF16)
    no(ea.EA_E_INVAL, table.lookup, ids, w, out=torch.empty(dim, 2, device="cuda").t())
    no(ea.EA_E_INVAL, table.grad, ids, dy[:1])
    no(ea.EA_E_INVAL, table.grad, ids, dy, accumulate=True)
    no(ea.EA_E_INVAL, table.grad, ids, dy, out=torch.empty(vocab, dim, device="cuda", dtype=torch.float64))
    no(ea.EA_E_INVAL, ea.Embedding, vocab, dim, 4, padding_idx=vocab)
    no(ea.EA_E_INVAL, ea.Embedding, vocab, dim, 4, padding_idx=-1)
    g = _randn(10, seed=82)
    norm = ea.GradNorm([10])
    no(ea.EA_E_INVAL, norm, [g[:9]])
    no(ea.EA_E_INVAL, norm, [g, g])
    no(ea.EA_E_INVAL, norm, [g.to(BF16)])
    no(ea.EA_E_INVAL, norm, [g.cpu()])
    no(ea.EA_E_INVAL, norm, [_randn(20, seed=1)[::2]])
    no(ea.EA_E_INVAL, norm, [g], max_norm=-1.0)
    no(ea.EA_E_INVAL, norm, [g], max_norm=float("nan"))
    no(ea.EA_E_INVAL, norm, [g], grad_scale=0.0)
    no(ea.EA_E_INVAL, norm, [g], out=torch.empty(3, device="cuda"))
    p = _randn(10, seed=83)
    opt = ea.AdamW([p])
    no(ea.EA_E_INVAL, opt.step, [g], lr=float("nan"))
    no(ea.EA_E_INVAL, opt.step, [g[:5]], lr=1e-3)
    no(ea.EA_E_INVAL, opt.step, [g], lr=1e-3, clip=torch.ones(1, device="cuda"))
    no(ea.EA_E_INVAL, opt.step, [g], lr=1e-3, clip=torch.ones(2))
    no(ea.EA_E_UNSUPPORTED, ea.AdamW, [p.half()])
    no(ea.EA_E_INVAL, ea.AdamW, [p], state_bits=16)
    no(ea.EA_E_INVAL, ea.AdamW, [p], betas=(1.0, 0.9))
    no(ea.EA_E_INVAL, ea.AdamW, [p], weight_decay=[0.1, 0.2])
    no(ea.EA_E_INVAL, ea.AdamW, [p], copies=[torch.empty(10, device="cuda")])
    no(ea.EA_E_INVAL, ea.AdamW, [p], states={"m": [torch.zeros(10, device="cuda")]})
    no(ea.EA_E_INVAL, ea.AdamW, [p], states={"m": [torch.zeros(10, device="cuda")], "v": [torch.zeros(9, device="cuda")]})
    no(ea.EA_E_INVAL, ea.AdamW, [])
    no(ea.EA_E_INVAL, ea.AdamW, [p, _randn(4, seed=1, dtype=BF16)])
    assert torch.equal(table.lookup(ids, w), w[ids])


def test_refusals_of_copies_and_states_that_are_no_tensors():
    p = _randn(10, seed=84)
    for bad in (dict(copies=[1.0]), dict(states={"m": [1.0], "v": [p.clone()]}), dict(states={"m": [p.clone()], "v": [None]})):
        with pytest.raises(ea.EAError) as ex:
            ea.AdamW([p], **bad)
        assert ex.value.status == ea.EA_E_INVAL and str(ex.value)
