"""The operators of include/ea_block.h on the GPU against plain implementations in 64 bits.

Tolerances come from the operators' own roundings: u = 2^-24 for each operation in binary32, half a unit in the last place for
the rounding to a 16-bit type, gamma_n = n u / (1 - n u) for a sum of n terms in any order (Higham, Accuracy and Stability of
Numerical Algorithms, Section 4.2), and of a gate 6 + 1.2 |z| units of 2^-23: the documented 2 and 1 of the approximate power
of two and reciprocal, 1.2 |z| of the exponent's product with log2 e, and the roundings of a sum and two products.  Products of
bounds (u^2 and the like) are covered by a factor of 1.01."""
import numpy as np
import pytest
import torch

import paper_2205_14473_gb300 as ea

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}     # relative, of normal values
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}      # spacing of subnormal values
PAIRS = [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]


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


def _randn(*shape, seed=0, dtype=F32, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * std + mean).to(dtype)


def _inside(got, want, bound, what, stored=None):
    """|got - want| <= bound, and what rounding to `stored` (default: got's type) adds."""
    stored = stored or got.dtype
    got, want, bound = got.double(), want.double(), bound.double() * 1.01
    bound = bound + HALF_ULP[stored] * (want.abs() + bound) + TINY[stored]
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        at = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {at}: {float(got[at])!r} for "
                             f"{float(want[at])!r} +- {float(bound[at])!r}")


def _gamma(n):
    return n * U / (1 - n * U)


def _off(t, k):
    """A copy of t whose address is k elements after a 256-byte boundary."""
    flat = torch.zeros(t.numel() + k, device="cuda", dtype=t.dtype)
    flat[k:] = t.flatten()
    return flat[k:].view(t.shape)


def _wide(t, before, after):
    """A copy of t whose rows are pieces of longer ones."""
    flat = torch.full((*t.shape[:-1], t.shape[-1] + before + after), 7.0, device="cuda", dtype=t.dtype)
    flat[..., before:before + t.shape[-1]] = t
    return flat[..., before:before + t.shape[-1]]


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def _no(status, f, *a, **k):
    with pytest.raises(ea.EAError) as ex:
        f(*a, **k)
    assert ex.value.status == status and str(ex.value)


# ------------------------------------------------------------------------------------------ layer norm

def _check_forward(y, stats, x, w, b, eps=1e-5):
    n, X = x.shape[-1], x.double()
    mean = X.mean(-1, keepdim=True)
    d = X - mean
    var = d.square().mean(-1, keepdim=True)
    e32 = float(np.float32(eps))
    rstd = (var + e32).rsqrt()
    e_mean = _gamma(n + 2) * X.abs().mean(-1, keepdim=True)
    e_var = (_gamma(n + 2) + 4 * U) * (var + e_mean ** 2) + e_mean ** 2
    e_rel = 0.5 * e_var / (var + e32) + 4 * U                  # of rstd: the root halves it; its own and eps's roundings
    w = torch.ones(n, device="cuda", dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(n, device="cuda", dtype=torch.float64) if b is None else b.double()
    want = d * rstd * w + b
    bound = w.abs() * rstd * (e_mean + d.abs() * (e_rel + 4 * U)) + U * ((d * rstd * w).abs() + want.abs())
    _inside(y, want, bound, "y")
    _inside(stats[..., :1], mean, e_mean, "mean")
    _inside(stats[..., 1:], rstd, rstd * e_rel, "rstd")


@pytest.mark.parametrize("shape", [(1,), (0,), (3, 0), (7,), (2, 33), (1, 257), (4, 3, 5), (1000,)])
@pytest.mark.parametrize("dim", [1, 3, 8, 64, 769, 1600])
def test_norm_shapes(shape, dim):
    x, w, b = _randn(*shape, dim, seed=1, mean=0.5), _randn(dim, seed=2), _randn(dim, seed=3)
    y, stats = ea.LayerNorm(dim, 1024).forward(x, w, b)
    assert y.shape == x.shape and stats.shape == (*shape, 2)
    _check_forward(y, stats, x, w, b)


# widths around every split of a row: packs, warps, CTAs, and past what registers hold
@pytest.mark.parametrize("dim", [2, 7, 31, 32, 33, 100, 255, 256, 257, 511, 512, 513, 1000, 1023, 1024, 1025, 1536, 2047, 2048, 2049, 2056, 4095,
                                 4096, 4104, 5003, 8191, 8192, 8193, 8200, 12_288, 16_384, 16_385, 20_000, 70_001, 100_000])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_norm_widths(dim, types):
    x, w, b = _randn(13, dim, seed=dim, mean=-0.3, dtype=types[0]), _randn(dim, seed=2), _randn(dim, seed=3)
    norm = ea.LayerNorm(dim, 13, eps=1e-6)
    y, stats = norm.forward(x, w, b)
    _check_forward(y, stats, x, w, b, 1e-6)
    dy, add = _randn(13, dim, seed=dim + 1, dtype=types[1]), _randn(13, dim, seed=dim + 2, dtype=types[0])
    _check_grad(norm.grad(dy, x, stats, w, add=add, dw=True, db=True), dy, x, stats, w, add)


@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("wt", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [40, 37, 1600])
def test_norm_types(xt, yt, wt, dim):
    x, w, b = _randn(300, dim, seed=4, dtype=xt), _randn(dim, seed=5, dtype=wt, mean=1.0), _randn(dim, seed=6, dtype=wt)
    norm = ea.LayerNorm(dim, 300)
    y, stats = norm.forward(x, w, b, dtype=yt)
    assert y.dtype == yt
    _check_forward(y, stats, x, w, b)
    dy, add = _randn(300, dim, seed=7, dtype=yt), _randn(300, dim, seed=8, dtype=xt)
    before = _randn(2, dim, seed=9, dtype=wt)
    out = before.clone()
    got = norm.grad(dy, x, stats, w, add=add, dw=out[0], db=out[1], accumulate=True)
    _check_grad(got, dy, x, stats, w, add, before)
    _check_grad(norm.grad(dy, x, stats, w, dw=out[0], db=out[1]), dy, x, stats, w)


def test_norm_without_weights():
    x, dy = _randn(50, 96, seed=10), _randn(50, 96, seed=11)
    w, b, norm = _randn(96, seed=12), _randn(96, seed=13), ea.LayerNorm(96, 50)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, stats = norm.forward(x, ww, bb)
        _check_forward(y, stats, x, ww, bb)
        for dw, db in ((None, None), (True, None), (None, True), (True, True)):
            got = norm.grad(dy, x, stats, ww, dw=dw, db=db)
            assert (got[1] is None) == (dw is None) and (got[2] is None) == (db is None)
            _check_grad(got, dy, x, stats, ww)


def test_norm_of_constant_rows_and_of_large_offsets():
    x = _randn(6, 100, seed=14)
    x[0], x[1], x[2] = 0.0, 3.0, -1e30
    x[3] += 1000.0
    x[4, 5] = 1e4
    y, stats = ea.LayerNorm(100, 6).forward(x)
    _check_forward(y, stats, x, None, None)
    assert (y[0] == 0).all() and float(stats[0, 1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)


def test_norm_keeps_nan_in_its_rows():
    x, dy, w = _randn(5, 200, seed=15), _randn(5, 200, seed=16), _randn(200, seed=17)
    x[1, 3], x[3, 199] = float("nan"), float("inf")
    norm = ea.LayerNorm(200, 5)
    y, stats = norm.forward(x, w)
    assert y[[1, 3]].isnan().all() and y[[0, 2, 4]].isfinite().all()
    dx, dw, db = norm.grad(dy, x, stats, w, dw=True, db=True)
    assert dx[[1, 3]].isnan().all() and dx[[0, 2, 4]].isfinite().all() and dw.isnan().all() and db.isfinite().all()


def _check_grad(got, dy, x, stats, w, add=None, before=None):
    n, dx, dw, db = x.shape[-1], *got
    mean, r = stats[..., :1].double(), stats[..., 1:].double()
    DY, t = dy.double(), (x.double() - mean) * r
    q = DY if w is None else DY * w.double()
    s, p = q.mean(-1, keepdim=True), (q * t).mean(-1, keepdim=True)
    want = r * (q - s - t * p)
    e_s, e_p = _gamma(n + 3) * q.abs().mean(-1, keepdim=True), _gamma(n + 6) * (q * t).abs().mean(-1, keepdim=True)
    bound = r * (U * q.abs() + e_s + t.abs() * e_p + 3 * U * (t * p).abs() + 3 * U * (q.abs() + s.abs() + (t * p).abs())) + 2 * U * want.abs()
    if add is not None:
        want = want + add.double()
        bound = bound + U * want.abs()
    _inside(dx, want, bound, "dx")
    rows = max(1, x.numel() // n)
    for k, (g, terms) in enumerate(((dw, DY * t), (db, DY))):
        if g is None:
            continue
        terms = terms.reshape(-1, n)
        want, bound = terms.sum(0), _gamma(rows + 3) * terms.abs().sum(0)
        if before is not None:
            want = want + before[k].double()
            bound = bound + U * want.abs()
        _inside(g, want, bound, ("dw", "db")[k])


# numbers of rows around every split of the sums over them
@pytest.mark.parametrize("rows", [1, 2, 3, 7, 8, 9, 31, 33, 100, 151, 152, 153, 303, 305, 607, 609, 1215, 1217, 2433, 5003, 20_011])
@pytest.mark.parametrize("dim", [1, 3, 8, 64, 515, 1600])
def test_norm_rows(rows, dim):
    x, dy, w = _randn(rows, dim, seed=rows, dtype=BF16, mean=0.1), _randn(rows, dim, seed=rows + 1, dtype=BF16), _randn(dim, seed=18)
    norm = ea.LayerNorm(dim, rows)
    y, stats = norm.forward(x, w, w)
    _check_forward(y, stats, x, w, w)
    got = norm.grad(dy, x, stats, w, dw=True, db=True)
    _check_grad(got, dy, x, stats, w)
    again = norm.grad(dy, x, stats, w, dw=torch.full_like(w, float("nan")), db=torch.full_like(w, float("nan")))
    assert all(_same(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dim", [64, 100, 1600, 2049])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_strided_rows(dim, dtype):
    """Batches in other orders, pieces of longer rows, rows off every boundary, one row in the place of many."""
    x, dy, add = (_randn(5, 9, dim, seed=20 + k, dtype=dtype) for k in range(3))
    w, b, norm = _randn(dim, seed=23), _randn(dim, seed=24), ea.LayerNorm(dim, 64)

    def views(t):
        yield t.transpose(0, 1).contiguous().transpose(0, 1)
        for k in (1, 2, 3, 8):
            yield _off(t, k)
            yield _wide(t, k, 5)
        yield _wide(t, 16, 16)
        yield t.transpose(0, 2).contiguous().transpose(0, 2)     # rows that are not contiguous
        yield t

    for a, c, e in zip(views(x), views(dy), views(add)):
        y, stats = norm.forward(a, w, b)
        _check_forward(y, stats, x, w, b)
        _check_grad(norm.grad(c, a, stats, w, add=e, dw=True, db=True), dy, x, stats, w, add)
    for k in (0, 1, 8):                                          # into pieces of longer rows, and nothing beside them
        wide, more = (torch.full((5, 11, dim + 16), 7.0, device="cuda", dtype=dtype) for _ in range(2))
        y, stats = norm.forward(x, w, b, out=wide[:, 1:-1, k:k + dim])
        _check_forward(y, stats, x, w, b)
        dx, _, _ = norm.grad(dy, x, stats, w, add=add, out=more[:, 1:-1, k:k + dim])
        _check_grad((dx, None, None), dy, x, stats, w, add)
        for t in (wide, more):
            t[:, 1:-1, k:k + dim] = 7.0
            assert (t == 7.0).all()
    one = dy[:1, :1].expand(5, 9, dim)
    _check_grad(norm.grad(one, x, stats, w, dw=True, db=True), one, x, stats, w)
    same = norm.forward(x[:1].expand(5, 9, dim), w, b)[0]
    assert _same(same[0], same[4])


@pytest.mark.parametrize("dim", [64, 77, 9000])
def test_norm_in_place(dim):
    x, dy, add = (_randn(33, dim, seed=25 + k, dtype=BF16) for k in range(3))
    w, norm = _randn(dim, seed=28), ea.LayerNorm(dim, 33)
    y, stats = norm.forward(x, w)
    z = x.clone()
    assert norm.forward(z, w, out=z)[0] is z and _same(z, y)
    want = norm.grad(dy, x, stats, w, add=add, dw=True, db=True)
    for k in range(3):
        c, a, e = dy.clone(), x.clone(), add.clone()
        got = norm.grad(c, a, stats, w, add=e, out=(c, a, e)[k], dw=True, db=True)
        assert all(_same(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dim,off", [(64, 0), (64, 1), (77, 0), (77, 3), (9000, 1)])
def test_norm_sums_alone(dim, off):
    """The C call without dx; what is named as added, at an address of its own, is not looked at."""
    from paper_2205_14473_gb300 import block_abi as A

    x, dy, add = _off(_randn(21, dim, seed=34, dtype=BF16), off), _off(_randn(21, dim, seed=35, dtype=BF16), off), _off(_randn(21, dim, seed=36, dtype=BF16), 1)
    norm = ea.LayerNorm(dim, 21)
    _, stats = norm.forward(x)
    dw, db = torch.empty(2, dim, device="cuda")
    c = A.ea_layernorm_call(1, 21, 0, dim, 0, dim, 0, 0, 0, dim, 1, 1, 0, 0)
    L = ea.lib()
    assert L.ea_layernorm_backward(norm.h, c, dy.data_ptr(), x.data_ptr(), stats.data_ptr(), None, add.data_ptr(), None, dw.data_ptr(), db.data_ptr(), 0) == 0
    want = norm.grad(dy, x, stats, dw=True, db=True)
    assert _same(dw, want[1]) and _same(db, want[2])
    assert L.ea_layernorm_backward(norm.h, c, dy.data_ptr(), x.data_ptr(), stats.data_ptr(), None, None, None, None, None, 0) == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("wt", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 100, 8200])
def test_norm_weights_at_any_address(wt, dim):
    """Pieces of flat vectors, off every boundary."""
    x, dy, w, b = _randn(9, dim, seed=37), _randn(9, dim, seed=38), _randn(dim, seed=39, dtype=wt), _randn(dim, seed=40, dtype=wt)
    norm, flat = ea.LayerNorm(dim, 9), torch.full((2 * dim + 9,), 7.0, device="cuda", dtype=wt)
    y, stats = norm.forward(x, w, b)
    for k in (1, 3, 4):
        assert _same(norm.forward(x, _off(w, k), _off(b, k + 1))[0], y)
        flat.fill_(7.0)
        got = norm.grad(dy, x, stats, _off(w, k), dw=flat[k:k + dim], db=flat[k + dim + 1:k + 2 * dim + 1])
        _check_grad(got, dy, x, stats, w)
        assert (flat[:k] == 7).all() and float(flat[k + dim]) == 7 and (flat[k + 2 * dim + 1:] == 7).all()


def test_norm_of_no_rows():
    norm, x, stats = ea.LayerNorm(8, 4), torch.zeros(0, 8, device="cuda"), torch.zeros(0, 2, device="cuda")
    dw, db = torch.full((2, 8), 3.0, device="cuda")
    dx, _, _ = norm.grad(x, x, stats, dw=dw, db=db, accumulate=True)
    assert dx.shape == (0, 8) and (dw == 3).all() and (db == 3).all()
    norm.grad(x, x, stats, dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()


def test_norm_gradient_against_differences():
    """<gradients, direction> against the central difference of sum(c y) along it, in 64 bits of y's formula on x moved by h
    in 32: the difference's own error is h^2 / 6 of the third derivative, below 1e-5 of the terms at h = 2^-7 and spreads near 1."""
    dim, rows, h = 24, 11, 2.0 ** -7
    x, w, b, c = _randn(rows, dim, seed=30), _randn(dim, seed=31), _randn(dim, seed=32), _randn(rows, dim, seed=33)
    norm = ea.LayerNorm(dim, rows)
    _, stats = norm.forward(x, w, b)
    dx, dw, db = norm.grad(c, x, stats, w, dw=True, db=True)

    def loss(x, w, b):
        x = x.double()
        d = x - x.mean(-1, keepdim=True)
        return float((c.double() * (d * (d.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w.double() + b.double())).sum())

    for k in range(4):
        ex, ew, eb = (torch.sign(_randn(*t.shape, seed=34 + 3 * k + i)).double() for i, t in enumerate((x, w, b)))
        quotient = (loss(x + h * ex, w + h * ew, b + h * eb) - loss(x - h * ex, w - h * ew, b - h * eb)) / (2 * h)
        exact = float((dx.double() * ex).sum() + (dw.double() * ew).sum() + (db.double() * eb).sum())
        size = float(dx.abs().sum() + dw.abs().sum() + db.abs().sum())
        assert abs(quotient - exact) <= size * (10 * h * h + 100 * U)


# ------------------------------------------------------------------------------------------ gated recurrence

def _gates(z):
    f = torch.sigmoid(z)
    return f, torch.sigmoid(-z), 2.0 ** -23 * (6 + 1.2 * z.abs())   # f, 1 - f, and the relative error of either


def _ends(lengths, batch, length):
    ends = torch.full((batch,), length, device="cuda") if lengths is None else lengths.long().clamp(0, length)
    return (torch.arange(length, device="cuda")[None] < ends[:, None])[..., None].double()


FLUSH = 2.0 ** -126  # gates below it may count as 0
ADDS = 64  # roundings of sums that a term meets beyond one for each row that it is carried through (pieces joined)


def _check_scan(h, final, z, v, initial=None, lengths=None):
    Z, V = z.double(), v.double()
    f, shut, rel = _gates(Z)
    batch, length, dim = z.shape
    inside = _ends(lengths, batch, length)
    x = torch.zeros(batch, dim, device="cuda", dtype=torch.float64) if initial is None else initial.double()
    size, err = x.abs(), torch.zeros_like(x)
    # a sequence's state stays as it is behind its end
    new = inside * shut * V
    fine, f = inside * (rel + 3 * U), inside * f + (1 - inside)
    flush = inside * FLUSH * (1 + V.abs())
    want, bound, sizes = torch.empty_like(Z), torch.empty_like(Z), new.abs()
    for t in range(length):
        kept = f[:, t] * size
        flushed = torch.addcmul(flush[:, t], inside[:, t] * FLUSH, size)
        size = torch.add(kept, sizes[:, t], out=sizes[:, t])
        err = torch.addcmul(torch.addcmul(flushed, f[:, t], err), fine[:, t], size, out=bound[:, t])
        x = torch.addcmul(new[:, t], f[:, t], x, out=want[:, t])
    want, bound = want * inside, (bound + ADDS * U * sizes) * inside
    _inside(h, want, bound, "h")
    assert (h.double() * (1 - inside) == 0).all()
    if final is not None:
        _inside(final, x, err + ADDS * U * size, "final")


def _check_scan_grad(got, dh, z, v, h, initial=None, lengths=None, d_final=None):
    Z, V, DH, H = z.double(), v.double(), dh.double(), h.double()
    f, shut, rel = _gates(Z)
    batch, length, dim = z.shape
    inside = _ends(lengths, batch, length)
    zero = torch.zeros(batch, dim, device="cuda", dtype=torch.float64)
    late = zero if d_final is None else d_final.double()       # f_{t+1} g_{t+1}
    size, err = late.abs(), torch.zeros_like(late)
    wants = [torch.zeros_like(Z) for _ in range(4)]
    for t in reversed(range(length)):
        k = inside[:, t]
        g, gsize, gerr = DH[:, t] + late, DH[:, t].abs() + size, err + U * (DH[:, t].abs() + size) + ADDS * U * (DH[:, t].abs() + size)
        before = H[:, t - 1] if t else zero if initial is None else initial.double()
        e = rel[:, t]
        d = before - V[:, t]
        wants[0][:, t] = k * shut[:, t] * g
        wants[1][:, t] = k * (shut[:, t] * (gerr + (e + 2 * U) * gsize) + FLUSH * (1 + gsize))
        wants[2][:, t] = k * f[:, t] * shut[:, t] * g * d
        wants[3][:, t] = k * (f[:, t] * shut[:, t] * d.abs() * (gerr + (2 * e + 5 * U) * gsize) + FLUSH * (2 + gsize) * (1 + d.abs()))
        nlate, nsize = f[:, t] * g, f[:, t] * gsize
        nerr = f[:, t] * (err + U * gsize) + (e + 3 * U) * nsize + FLUSH * (1 + gsize)
        late, size, err = k * nlate + (1 - k) * late, k * nsize + (1 - k) * size, k * nerr + (1 - k) * err
    dz, dv, d_initial = got
    _inside(dv, wants[0], wants[1], "dv")
    _inside(dz, wants[2], wants[3], "dz")
    assert (dz.double() * (1 - inside) == 0).all() and (dv.double() * (1 - inside) == 0).all()
    if d_initial is not None:
        _inside(d_initial, late, err + ADDS * U * size, "d_initial")


def _scan_inputs(batch, length, dim, dtype=F32, seed=0, mean=1.0):
    z, v, dh = (_randn(batch, length, dim, seed=40 + 5 * seed + k, dtype=dtype, mean=mean if k == 0 else 0.0, std=1.5 if k == 0 else 1.0)
                for k in range(3))
    return z, v, dh, _randn(batch, dim, seed=43 + 5 * seed), _randn(batch, dim, seed=44 + 5 * seed)


def _check_both(scan, z, v, dh, initial=None, d_final=None, lengths=None):
    h, final = scan.forward(z, v, initial=initial, lengths=lengths, final=True)
    _check_scan(h, final, z, v, initial, lengths)
    got = scan.grad(dh, z, v, h, initial=initial, lengths=lengths, d_final=d_final, d_initial=True)
    _check_scan_grad(got, dh, z, v, h, initial, lengths, d_final)
    return h, final, got


# lengths around every split of a sequence
@pytest.mark.parametrize("length", [0, 1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 1000,
                                    1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 5003])
@pytest.mark.parametrize("batch,dim,dtype", [(2, 64, BF16), (3, 40, F32), (1, 37, F16)])
def test_scan_lengths(length, batch, dim, dtype):
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=length)
    _check_both(ea.GatedScan(dim), z, v, dh, first, last)


@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 32, 33, 56, 63, 64, 65, 72, 100, 127, 128, 129, 515, 768, 1600, 2049])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,length", [(1, 700), (7, 50)])
def test_scan_widths(dim, dtype, batch, length):
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=dim)
    _check_both(ea.GatedScan(dim), z, v, dh, first, last)


@pytest.mark.parametrize("batch,length,dim", [(300, 65, 64), (1000, 3, 24), (20, 400, 1600), (40, 300, 515), (2, 9000, 256), (1, 12_001, 8), (600, 130, 512)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scan_batches(batch, length, dim, dtype):
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=3)
    scan = ea.GatedScan(dim)
    h, final, got = _check_both(scan, z, v, dh, first, last)
    again = scan.forward(z, v, initial=first, final=True)
    assert _same(again[0], h) and _same(again[1], final)
    assert all(_same(a, b) for a, b in zip(got, scan.grad(dh, z, v, h, initial=first, d_final=last, d_initial=True)))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("state", [False, True])
def test_scan_without_states(dtype, state):
    z, v, dh, first, last = _scan_inputs(3, 130, 72, dtype, seed=4)
    scan = ea.GatedScan(72)
    first, last = (first, None) if state else (None, last)
    h, none = scan.forward(z, v, initial=first)
    assert none is None
    _check_scan(h, None, z, v, first)
    got = scan.grad(dh, z, v, h, initial=first, d_final=last)
    assert got[2] is None
    _check_scan_grad(got, dh, z, v, h, first, None, last)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("length,dim", [(300, 64), (1100, 33), (2500, 16), (65, 256)])
def test_scan_of_ragged_batches(dtype, length, dim):
    """Lengths of zero, one, all rows and around the splits; what lies behind them is NaN and not looked at."""
    ends = torch.tensor([0, 1, length, length - 1, 63, 64, 65, length // 2, 0, 17], device="cuda").clamp(max=length)
    z, v, dh, first, last = _scan_inputs(ends.numel(), length, dim, seed=5)
    behind = torch.arange(length, device="cuda")[None] >= ends[:, None]
    scan, lengths = ea.GatedScan(dim), ends.to(dtype)
    for t in (z, v, dh):
        t[behind] = float("nan")
    h, final = scan.forward(z, v, initial=first, lengths=lengths, final=True)
    clean = [t.nan_to_num(0.0) for t in (z, v, dh)]
    _check_scan(h, final, clean[0], clean[1], first, lengths)
    assert _same(final[0], first[0]) and _same(final[8], first[8])
    h[behind] = float("nan")
    got = scan.grad(dh, z, v, h, initial=first, lengths=lengths, d_final=last, d_initial=True)
    _check_scan_grad(got, clean[2], clean[0], clean[1], h.nan_to_num(0.0), first, lengths, last)
    assert _same(got[2][0], last[0])
    scan.sync()


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_lengths_outside_the_rows(dtype):
    z, v, dh, first, last = _scan_inputs(4, 70, 24, seed=6)
    scan = ea.GatedScan(24)
    lengths = torch.tensor([-3, 71, 2 ** 31 - 1, 12], device="cuda", dtype=dtype)
    if dtype == torch.int64:
        lengths[2] = 2 ** 32 + 5                                # not 5
    h, final = scan.forward(z, v, initial=first, lengths=lengths, final=True)
    _check_scan(h, final, z, v, first, lengths)
    with pytest.raises(ea.EAError) as ex:
        scan.sync()
    assert ex.value.status == ea.EA_E_DEVICE_CHECK
    scan.sync()
    _check_scan_grad(scan.grad(dh, z, v, h, initial=first, lengths=lengths, d_final=last, d_initial=True), dh, z, v, h, first, lengths, last)
    with pytest.raises(ea.EAError):
        scan.sync()
    scan.forward(z, v, lengths=lengths[3:].expand(4))
    scan.sync()


def test_gates_at_their_ends():
    """f or 1 - f of 1 and 0, and gates far out; infinite gates hold or replace the state."""
    z = torch.tensor([0.0, 20.0, -20.0, 88.0, -88.0, 100.0, -100.0, 1000.0, -1000.0, float("inf"), float("-inf")], device="cuda")
    batch, length, dim = 2, 40, z.numel()
    v = _randn(batch, length, dim, seed=50)
    first = _randn(batch, dim, seed=51)
    scan, Z = ea.GatedScan(dim), z.expand(batch, length, dim)
    h, final = scan.forward(Z, v, initial=first, final=True)
    _check_scan(h[..., :9], final[:, :9], Z[..., :9], v[..., :9], first[:, :9].contiguous())
    assert _same(final[:, 9], first[:, 9]) and _same(final[:, 10], v[:, -1, 10])
    dh = _randn(batch, length, dim, seed=52)
    got = scan.grad(dh, Z, v, h, initial=first, d_initial=True)
    _check_scan_grad([g[..., :9] for g in got], dh[..., :9], Z[..., :9], v[..., :9], h[..., :9], first[:, :9])
    assert (got[0][..., 9:] == 0).all() and (got[1][..., 9] == 0).all() and _same(got[1][..., 10], dh[..., 10])


def test_scan_keeps_nan_where_it_arises():
    z, v, _, first, _ = _scan_inputs(2, 200, 16, seed=7)
    v[0, 50, 3], z[1, 100, 5] = float("nan"), float("nan")
    h, _ = ea.GatedScan(16).forward(z, v, initial=first)
    want = torch.zeros_like(h, dtype=torch.bool)
    want[0, 50:, 3], want[1, 100:, 5] = True, True
    assert torch.equal(h.isnan(), want)


@pytest.mark.parametrize("dim", [64, 96, 33, 1600])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,length", [(2, 333), (9, 40)])
def test_scan_of_strided_rows(dim, dtype, batch, length):
    """Halves of one product, time before batch, rows off every boundary, one sequence in the place of many."""
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=8)
    scan = ea.GatedScan(dim)
    h, final, got = _check_both(scan, z, v, dh, first, last)

    def by_time(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    def check(zz, vv, hh, gg, **out):
        a = scan.forward(zz, vv, initial=first, final=True)
        b = scan.grad(gg, zz, vv, hh, initial=first, d_final=last, d_initial=True, **out)
        _check_scan(a[0], a[1], z, v, first)
        _check_scan_grad(b, dh, z, v, h, first, None, last)

    half = torch.cat([z, v], 2)
    check(half[..., :dim], half[..., dim:], h, dh)
    check(by_time(z), by_time(v), by_time(h), by_time(dh), dz=by_time(z), dv=by_time(v))
    for k in (1, 2, 4):
        check(_off(z, k), v, _off(h, k), dh)
        check(_wide(z, k, 3), _wide(v, 0, 8), h, _wide(dh, 8, k))
    check(z.transpose(1, 2).contiguous().transpose(1, 2), v, h, dh)  # rows that are not contiguous
    both, more = (torch.full((batch, length + 2, 2 * dim + 8), 7.0, device="cuda", dtype=dtype) for _ in range(2))
    for k in (0, 1, 8):
        scan.grad(dh, z, v, h, initial=first, d_final=last, dz=both[:, 1:-1, k:k + dim], dv=both[:, 1:-1, dim + k:2 * dim + k])
        scan.forward(z, v, initial=first, out=more[:, 1:-1, k:k + dim])
        _check_scan_grad((both[:, 1:-1, k:k + dim], both[:, 1:-1, dim + k:2 * dim + k], None), dh, z, v, h, first, None, last)
        _check_scan(more[:, 1:-1, k:k + dim], None, z, v, first)
        both[:, 1:-1, k:2 * dim + k] = 7.0
        more[:, 1:-1, k:k + dim] = 7.0
        assert (both == 7).all() and (more == 7).all()
    one = z[:1].expand(batch, length, dim)
    a = scan.forward(one, v, initial=first, final=True)
    _check_scan(a[0], a[1], one, v, first)
    sums = torch.ones((), device="cuda", dtype=dtype).expand(batch, length, dim)  # the gradient of h.sum()
    _check_scan_grad(scan.grad(sums, z, v, h, initial=first), sums, z, v, h, first)


@pytest.mark.parametrize("length", [1, 40, 700])
@pytest.mark.parametrize("dim", [64, 33])
def test_scan_in_place(length, dim):
    z, v, dh, first, last = _scan_inputs(3, length, dim, BF16, seed=9)
    scan = ea.GatedScan(dim)
    h, final = scan.forward(z, v, initial=first, final=True)
    for k in range(2):
        a, b, s = z.clone(), v.clone(), first.clone()
        out, end = scan.forward(a, b, initial=s, out=(a, b)[k], final=s)
        assert end is s and _same(out, h) and _same(s, final)
    want = scan.grad(dh, z, v, h, initial=first, d_final=last, d_initial=True)
    for which in ((0, 1), (0, 2), (2, 1)):
        a = [z.clone(), v.clone(), dh.clone()]
        e = last.clone()
        got = scan.grad(a[2], a[0], a[1], h, initial=first, d_final=e, dz=a[which[0]], dv=a[which[1]], d_initial=e)
        assert all(_same(p, q) for p, q in zip(got, want))
    _no(ea.EA_E_INVAL, scan.grad, dh, z, v, h, dz=h)
    _no(ea.EA_E_INVAL, scan.grad, dh, z, v, h, dz=z, dv=z)


@pytest.mark.parametrize("batch", [1, 3, 64, 1000])
@pytest.mark.parametrize("dim", [8, 33, 1600])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_steps(batch, dim, dtype):
    """Row after row: the same as all rows at once, in a state of 32 bits."""
    length = 5
    z, v, _, first, _ = _scan_inputs(batch, length, dim, dtype, seed=10)
    scan, state = ea.GatedScan(dim), first.clone()
    rows = [scan.step(z[:, t], v[:, t], state) for t in range(length)]
    _check_scan(torch.stack(rows, 1), state, z, v, first)
    out = torch.empty(batch, dim, device="cuda", dtype=dtype)
    again = first.clone()
    assert scan.step(z[:, 0], v[:, 0], again, out=out) is out and _same(out, rows[0])


def test_pieces_of_a_sequence():
    """Two calls, the second from the first one's last states, and their gradients: as one call."""
    z, v, dh, first, last = _scan_inputs(3, 500, 48, seed=11)
    scan = ea.GatedScan(48)
    cut = 201
    a, mid = scan.forward(z[:, :cut], v[:, :cut], initial=first, final=True)
    b, end = scan.forward(z[:, cut:], v[:, cut:], initial=mid, final=True)
    h = torch.cat([a, b], 1)
    _check_scan(h, end, z, v, first)
    late = scan.grad(dh[:, cut:], z[:, cut:], v[:, cut:], b, initial=mid, d_final=last, d_initial=True)
    early = scan.grad(dh[:, :cut], z[:, :cut], v[:, :cut], a, initial=first, d_final=late[2], d_initial=True)
    _check_scan_grad((torch.cat([early[0], late[0]], 1), torch.cat([early[1], late[1]], 1), early[2]), dh, z, v, h, first, None, last)


@pytest.mark.parametrize("length", [0, 1, 5, 40, 700])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_states_at_any_address(length, dtype):
    """States that lie at no more than their element's boundary, and no sequences at all."""
    z, v, dh, first, last = _scan_inputs(3, length, 64, dtype, seed=13)
    scan = ea.GatedScan(64)
    h, final, got = _check_both(scan, z, v, dh, first, last)
    for k in (1, 2, 3):
        state, late = _off(first, k), _off(last, k)
        out = scan.forward(z, v, initial=state, final=state)
        _check_scan(out[0], out[1], z, v, first)
        back = scan.grad(dh, z, v, h, initial=_off(first, k), d_final=late, d_initial=late)
        _check_scan_grad(back, dh, z, v, h, first, None, last)
    none, end = scan.forward(z[:0], v[:0], final=True)
    assert none.shape == (0, length, 64) and end.shape == (0, 64)
    assert scan.grad(dh[:0], z[:0], v[:0], h[:0], d_initial=True)[2].shape == (0, 64)


def test_scan_gradient_against_differences():
    """As for the norm: central differences of sum(c h) + sum(e final) in 64 bits along random signs."""
    batch, length, dim, step = 2, 30, 5, 2.0 ** -8
    z, v, c, first, e = _scan_inputs(batch, length, dim, seed=12)
    scan = ea.GatedScan(dim)
    h, _ = scan.forward(z, v, initial=first)
    dz, dv, d0 = scan.grad(c, z, v, h, initial=first, d_final=e, d_initial=True)

    def loss(z, v, x):
        f, v, x, total = torch.sigmoid(z.double()), v.double(), x.double(), 0.0
        for t in range(length):
            x = f[:, t] * x + (1 - f[:, t]) * v[:, t]
            total += float((x * c[:, t].double()).sum())
        return total + float((x * e.double()).sum())

    for k in range(4):
        ez, ev, e0 = (torch.sign(_randn(*t.shape, seed=60 + 3 * k + i)) for i, t in enumerate((z, v, first)))
        quotient = (loss(z + step * ez, v + step * ev, first + step * e0) - loss(z - step * ez, v - step * ev, first - step * e0)) / (2 * step)
        exact = float((dz.double() * ez).sum() + (dv.double() * ev).sum() + (d0.double() * e0).sum())
        size = float(dz.abs().sum() + dv.abs().sum() + d0.abs().sum())
        assert abs(quotient - exact) <= size * (50 * step * step + 2000 * U)


# ------------------------------------------------------------------------------------------ dropout

def _halves(n, seed, counter):
    """The half words of elements 0 .. n - 1: Philox4x32-10 in numpy."""
    m = np.uint64(0xFFFFFFFF)
    j = np.arange(-(-n // 8), dtype=np.uint64)
    c = [j & m, j >> np.uint64(32), np.full_like(j, counter % 2 ** 32), np.full_like(j, counter >> 32)]
    k = [seed % 2 ** 32, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack(c, 1)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 2).reshape(-1)[:n].astype(np.int64)


def test_the_generator_is_philox():
    """The first known answer of Salmon et al.'s tests (counter and key 0)."""
    assert [int(a) | int(b) << 16 for a, b in _halves(8, 0, 0).reshape(4, 2)] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]


def _check_drop(y, x, p, seed, counter, add=None):
    limit = round(65536 * p)
    kept = torch.from_numpy(_halves(x.numel(), seed, counter) >= limit).cuda().view(x.shape)
    want = torch.where(kept, x.double(), 0.0) * (65536 / (65536 - limit) if limit < 65536 else 0.0)
    bound = 2 * U * want.abs()
    if add is not None:
        want = want + add.double()
        bound = bound + U * want.abs()
    _inside(y, want, bound, "dropout")
    if add is None:
        assert (torch.where(kept, 0.0, y.double()) == 0).all()


@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (0,), (3, 0), (0, 5), (5, 1), (33, 8), (2, 3, 5), (2, 100, 64), (3, 7, 33), (2, 2, 3, 24), (1_000_003,),
                                   (1001, 1000), (3, 5000, 72)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_shapes(shape, residual):
    x = _randn(*shape, seed=70)
    add = _randn(*shape, seed=71) if residual else None
    drop = ea.Dropout(0.1, seed=5)
    y = drop(x, 9, residual=add)
    _check_drop(y, x, 0.1, 5, 9, add)
    assert _same(drop.grad(x, 9), drop(x, 9))


@pytest.mark.parametrize("xt,yt", PAIRS + [(BF16, F32), (F16, F32)])
@pytest.mark.parametrize("shape", [(40, 64), (41, 37), (5, 9, 24)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_types(xt, yt, shape, residual):
    x, add = _randn(*shape, seed=72, dtype=xt), _randn(*shape, seed=73, dtype=yt) if residual else None
    y = ea.Dropout(0.3, seed=1)(x, 2, residual=add, dtype=yt)
    assert y.dtype == yt
    _check_drop(y, x, 0.3, 1, 2, add)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.05, 0.5, 0.9, 1 - 2.0 ** -16, 1.0])
@pytest.mark.parametrize("seed,counter", [(0, 0), (2 ** 64 - 1, 2 ** 64 - 1), (0x123456789ABCDEF, 2 ** 32), (7, 2 ** 32 - 1)])
def test_dropout_probabilities_and_counters(p, seed, counter):
    x = _randn(50, 100, seed=74)
    drop = ea.Dropout(p, seed=seed)
    y = drop(x, counter)
    assert drop.p == round(65536 * p) / 65536
    _check_drop(y, x, p, seed, counter)
    if counter < 2 ** 63:
        assert _same(drop(x, torch.tensor([counter], device="cuda")), y)
    if p == 1.0:
        assert (y == 0).all()
    if p < 2.0 ** -16:
        assert _same(y, x)


def test_dropped_infinities_leave_nothing():
    x, add = _randn(4000, seed=75), _randn(4000, seed=76)
    drop = ea.Dropout(0.5, seed=3)
    kept = drop(torch.ones_like(x), 1) != 0
    bad = x.clone()
    bad[~kept] = float("nan")
    bad[:2000][~kept[:2000]] = float("inf")
    assert _same(drop(bad, 1), drop(x, 1)) and _same(drop(bad, 1, residual=add), drop(x, 1, residual=add))
    x[kept] = float("-inf")
    y = drop(x, 1)
    assert (y[kept] == float("-inf")).all() and (y[~kept] == 0).all()


@pytest.mark.parametrize("dim", [64, 100, 37])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_of_strided_rows(dim, dtype):
    """The mask goes by the element's place in the shape: any strides and alignment give the same values."""
    x, add = _randn(4, 11, dim, seed=77, dtype=dtype), _randn(4, 11, dim, seed=78, dtype=dtype)
    drop = ea.Dropout(0.2, seed=4)
    want = drop(x, 3, residual=add)
    _check_drop(want, x, 0.2, 4, 3, add)
    for f in (lambda t: t.transpose(0, 1).contiguous().transpose(0, 1), lambda t: _off(t, 1), lambda t: _off(t, 4), lambda t: _wide(t, 1, 2),
              lambda t: _wide(t, 8, 16), lambda t: t.transpose(0, 2).contiguous().transpose(0, 2), lambda t: t.reshape(2, 2, 11, dim)):
        assert _same(drop(f(x), 3, residual=f(add)).reshape(x.shape), want)
        assert _same(drop(x, 3, residual=add, out=f(add)).reshape(x.shape), want) if f(x).stride(-1) == 1 and f(x).dim() == 3 else True
    for k in (0, 1, 8):
        wide = torch.full((4, 13, dim + 16), 7.0, device="cuda", dtype=dtype)
        assert _same(drop(x, 3, residual=add, out=wide[:, 1:-1, k:k + dim]), want)
        wide[:, 1:-1, k:k + dim] = 7.0
        assert (wide == 7).all()
    one = add[:1, :1].expand(4, 11, dim)
    _check_drop(drop(x, 3, residual=one), x, 0.2, 4, 3, one)
    a, b = x.clone(), add.clone()
    assert _same(drop(a, 3, residual=b, out=a), want)
    assert _same(drop(x, 3, residual=b, out=b), want)


def test_dropout_rates():
    """Of 2^22 elements the dropped ones lie within six standard deviations of p, in every one of the eight places of a block, and
    masks of two counters are unlike."""
    n, p = 1 << 22, 0.1
    drop, one = ea.Dropout(p, seed=11), torch.ones(1 << 22, device="cuda", dtype=BF16)
    a, b = (drop(one, k) == 0 for k in (0, 1))
    q = drop.p
    assert abs(float(a.double().mean()) - q) < 6 * (q * (1 - q) / n) ** 0.5
    assert ((a.view(-1, 8).double().mean(0) - q).abs() < 6 * (8 * q * (1 - q) / n) ** 0.5).all()
    assert abs(float((a & b).double().mean()) - q * q) < 6 * (q * q / n) ** 0.5


# ------------------------------------------------------------------------------------------ offsets beyond 2^31 elements

FAR = 2 ** 31 + 4096


def test_far_rows():
    """Rows that lie more than 2^31 elements apart, of every operator."""
    dim = 64
    flat, other = (torch.zeros(FAR + 8 * dim, device="cuda", dtype=BF16) for _ in range(2))
    far, to = (t.as_strided((2, 3, dim), (2 ** 31, dim, 1)) for t in (flat, other))
    x, v, dh = (_randn(2, 3, dim, seed=80 + k, dtype=BF16) for k in range(3))
    norm, scan, drop, w = ea.LayerNorm(dim, 6), ea.GatedScan(dim), ea.Dropout(0.1), _randn(dim, seed=83)
    far.copy_(x)
    y, stats = norm.forward(x, w)
    assert _same(norm.forward(far, w, out=to)[0], y)
    want = norm.grad(dh, x, stats, w, dw=True, db=True)
    assert all(_same(a, b) for a, b in zip(norm.grad(dh, far, stats, w, out=to, dw=True, db=True), want))
    assert _same(drop(far, 1, out=to), drop(x, 1))
    h, final = scan.forward(x, v, final=True)
    assert all(_same(a, b) for a, b in zip(scan.forward(far, v, out=to, final=True), (h, final)))
    want = scan.grad(dh, x, v, h)
    assert all(_same(a, b) for a, b in zip(scan.grad(dh, far, v, h, dz=to)[:2], want[:2]))
    far, to = (t.as_strided((1, 2, dim), (dim, 2 ** 31, 1)) for t in (flat, other))
    far.copy_(x[:1, :2])
    assert _same(scan.forward(far, v[:1, :2], out=to)[0], scan.forward(x[:1, :2], v[:1, :2])[0])
    assert _same(norm.forward(far, w, out=to)[0], y[:1, :2])


def test_many_elements():
    """More than 2^31 elements in one call: a stretch at either end and around 2^31."""
    dim = 512
    rows = FAR // dim
    x = torch.zeros(rows, dim, device="cuda", dtype=BF16)
    parts = [slice(0, 40), slice(2 ** 31 // dim - 20, 2 ** 31 // dim + 4), slice(rows - 4, rows)]
    for p in parts:
        x[p] = _randn(p.stop - p.start, dim, seed=p.start % 1000, dtype=BF16)
    norm, w = ea.LayerNorm(dim, rows), _randn(dim, seed=84)
    y, stats = norm.forward(x, w)
    for p in parts:
        _check_forward(y[p], stats[p], x[p], w, None)
    dx, _, db = norm.grad(x, x, stats, w, out=y, dw=True, db=True)
    for p in parts:
        _check_grad((dx[p], None, None), x[p], x[p], stats[p], w)
    terms = torch.cat([x[p] for p in parts]).double()
    _inside(db, terms.sum(0), _gamma(rows) * terms.abs().sum(0), "db")
    drop = ea.Dropout(0.25, seed=2)
    drop(x, 1, out=y)
    for p in parts:
        kept = torch.from_numpy(_halves_at(p.start * dim, (p.stop - p.start) * dim, 2, 1) >= 16384).cuda().view(-1, dim)
        want = torch.where(kept, x[p].float() * np.float32(65536 / 49152).item(), 0.0).to(BF16)
        assert _same(y[p], want)
    scan = ea.GatedScan(dim)
    z = x[None]
    h, final = scan.forward(z, z, out=y[None], final=True)
    state = torch.zeros(1, dim, device="cuda")
    at = 0
    for p in parts:                                             # between them f = 1/2: what was there is gone after 2^8 rows
        state.mul_(0.5 ** min(1000, p.start - at))
        _check_scan(h[:, p], None, z[:, p], z[:, p], state)
        state, at = scan.forward(z[:, p], z[:, p], initial=state, final=True)[1], p.stop
    _inside(final, state, 1e-5 * state.abs() + 1e-30, "final")  # re-associated: 64 u is 4e-6


def _halves_at(first, n, seed, counter):
    """As _halves, of elements first .. first + n - 1 (first a multiple of 8)."""
    m = np.uint64(0xFFFFFFFF)
    j = np.arange(first // 8, (first + n) // 8, dtype=np.uint64)
    c = [j & m, j >> np.uint64(32), np.full_like(j, counter % 2 ** 32), np.full_like(j, counter >> 32)]
    k = [seed % 2 ** 32, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack(c, 1)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 2).reshape(-1).astype(np.int64)


# ------------------------------------------------------------------------------------------ streams, graphs, refusals

class _Together:
    """The three as a residual block without its products: x + drop(scan(z(y), y)), y = norm(x), and the way back."""

    def __init__(self, batch, length, dim):
        self.norm, self.scan, self.drop = ea.LayerNorm(dim, batch * length), ea.GatedScan(dim), ea.Dropout(0.2, seed=6)

    def __call__(self, x, w, b, dout, counter):
        y, stats = self.norm.forward(x, w, b)
        h, _ = self.scan.forward(y, x)
        out = self.drop(h, counter, residual=x)
        dh = self.drop.grad(dout, counter)
        dz, dv, _ = self.scan.grad(dh, y, x, h)
        dx, dw, db = self.norm.grad(dz, x, stats, w, add=dout + dv, dw=True, db=True)
        return out, dx, dw, db


def test_a_block_and_its_gradient_against_autograd():
    """All three together: against autograd in 64 bits with the same mask.  A hundred and fifty operations in 32 bits on the
    longest path (30 rows of five, and the norm's), each 4 u of the largest value it meets at most: 600 u, twice."""
    batch, length, dim = 3, 30, 40
    x, dout, w, b = _randn(batch, length, dim, seed=90), _randn(batch, length, dim, seed=91), _randn(dim, seed=92, mean=1.0, std=0.1), _randn(dim, seed=93)
    block = _Together(batch, length, dim)
    got = block(x, w, b, dout, 12)
    X, W, B = (t.double().requires_grad_() for t in (x, w, b))
    d = X - X.mean(-1, keepdim=True)
    y = d * (d.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * W + B
    f, state, rows = torch.sigmoid(y), torch.zeros(batch, dim, device="cuda", dtype=torch.float64), []
    for t in range(length):
        state = f[:, t] * state + (1 - f[:, t]) * X[:, t]
        rows.append(state)
    kept = torch.from_numpy(_halves(x.numel(), 6, 12) >= round(65536 * 0.2)).cuda().view(x.shape)
    out = X + torch.stack(rows, 1) * kept * 65536 / (65536 - round(65536 * 0.2))
    out.backward(dout.double())
    for g, want in zip(got, (out.detach(), X.grad, W.grad, B.grad)):
        assert float((g.double() - want).abs().max()) <= 1200 * U * float(want.abs().max())


def test_another_current_stream():
    batch, length, dim = 4, 200, 128
    x, dout, w, b = _randn(batch, length, dim, seed=94), _randn(batch, length, dim, seed=95), _randn(dim, seed=96), _randn(dim, seed=97)

    def run(stream):
        block = _Together(batch, length, dim)
        torch.cuda.synchronize()
        out = []
        for t in range(5):
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                out += [y.clone() for y in block(x * (t + 1), w, b, dout, t)]
        torch.cuda.synchronize()
        return out

    assert all(_same(x, y) for x, y in zip(run(None), run(torch.cuda.Stream())))


def test_graphs_draw_by_a_counter_on_the_device():
    batch, length, dim = 3, 150, 96
    x, dout, w, b = _randn(batch, length, dim, seed=98), _randn(batch, length, dim, seed=99), _randn(dim, seed=100), _randn(dim, seed=101)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        block, counter = _Together(batch, length, dim), torch.zeros(1, device="cuda", dtype=torch.int64)
        block(x, w, b, dout, counter)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = block(x, w, b, dout, counter)
        counter.add_(1)
    plain = _Together(batch, length, dim)
    for t in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(_same(a, c) for a, c in zip(got, plain(x, w, b, dout, t)))
    assert int(counter) == 4


def test_written_tensors_count_as_modified():
    dim = 8
    x, w, state = _randn(2, 3, dim, seed=102), _randn(dim, seed=103), _randn(2, dim, seed=104)
    norm, scan, drop = ea.LayerNorm(dim, 6), ea.GatedScan(dim), ea.Dropout(0.1)
    y, stats = norm.forward(x, w)
    out, more, dw, db, st = torch.empty_like(x), torch.empty_like(x), torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda"), torch.empty_like(stats)
    for f, written in ((lambda: norm.forward(x, w, out=out, stats=st), (out, st)),
                       (lambda: norm.grad(x, x, stats, w, out=out, dw=dw, db=db), (out, dw, db)),
                       (lambda: scan.forward(x, x, out=out, final=state), (out, state)), (lambda: scan.step(x[:, 0], x[:, 0], state), (state,)),
                       (lambda: scan.grad(x, x, x, x, dz=out, dv=more, d_initial=state), (out, more, state)),
                       (lambda: drop(x, 1, out=out), (out,)), (lambda: drop.grad(x, 1, out=out), (out,))):
        for t in written:
            leaf = torch.ones_like(t, requires_grad=True)
            loss = (leaf * t).sum()
            f()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    p = torch.nn.Parameter(x.clone())
    assert not any(t.requires_grad for t in (norm.forward(p)[0], scan.forward(p, p)[0], drop(p, 1)))


def test_refusals():
    dim = 8
    x, w, stats = _randn(2, 3, dim, seed=105), _randn(dim, seed=106), torch.zeros(2, 3, 2, device="cuda")
    norm, scan, drop, bad = ea.LayerNorm(dim, 6), ea.GatedScan(dim), ea.Dropout(0.1), ea.EA_E_INVAL
    y, stats = norm.forward(x, w)
    h, _ = scan.forward(x, x)
    state = torch.zeros(2, dim, device="cuda")
    turned = _randn(dim, 3, 2, seed=107).permute(2, 1, 0)
    for f, a, k in (
            (norm.forward, (_randn(7, dim),), {}),                                  # more than max_rows
            (norm.forward, (x.cpu(),), {}), (norm.forward, (None,), {}), (norm.forward, (x[..., :7],), {}), (norm.forward, (x.double(),), {}),
            (norm.forward, (x, w[:7]), {}), (norm.forward, (x, w.double()), {}), (norm.forward, (x, w.cpu()), {}), (norm.forward, (x, w, w.half()), {}),
            (norm.forward, (x, w[:1].expand(dim)), {}), (norm.forward, (x,), dict(out=y[:1])), (norm.forward, (x,), dict(out=turned)),
            (norm.forward, (x,), dict(out=y, dtype=BF16)), (norm.forward, (x,), dict(dtype=torch.float64)), (norm.forward, (x,), dict(stats=stats[:1])),
            (norm.forward, (x,), dict(out=y[:1].expand(2, 3, dim))), (norm.forward, (x,), dict(out=y.flatten().as_strided((2, 3, dim), (24, 4, 1)))),
            (norm.forward, (x,), dict(out=torch.empty(100, device="cuda").as_strided((2, 3, dim), (20, 8, 1)))),
            (norm.grad, (x[:1], x, stats), {}), (norm.grad, (x, x, stats[..., :1]), {}), (norm.grad, (x, x, stats.half()), {}),
            (norm.grad, (x, x, stats), dict(add=x.half())), (norm.grad, (x, x, stats), dict(add=x[:1])), (norm.grad, (x, x, stats), dict(dw=w.double())),
            (norm.grad, (x, x, stats), dict(dw=w, db=w.half())), (norm.grad, (x, x, stats), dict(dw=True, accumulate=True)),
            (norm.grad, (x, x, stats), dict(dw=w, db=w)), (norm.grad, (x, x, stats), dict(dw=w[:7])), (norm.grad, (x, x, stats), dict(out=y.half())),
            (scan.forward, (x[0], x[0]), {}), (scan.forward, (x, x[:1]), {}), (scan.forward, (x, x.half()), {}), (scan.forward, (x.cpu(), x), {}),
            (scan.forward, (x, None), {}), (scan.forward, (x, x), dict(initial=state[:1])), (scan.forward, (x, x), dict(initial=state.half())),
            (scan.forward, (x, x), dict(final=state.half())), (scan.forward, (x, x), dict(final=state.t().contiguous().t())),
            (scan.forward, (x, x), dict(lengths=torch.ones(2, device="cuda"))), (scan.forward, (x, x), dict(lengths=torch.ones(3, device="cuda", dtype=torch.int64))),
            (scan.forward, (x, x), dict(lengths=torch.ones(2, dtype=torch.int64))), (scan.forward, (x, x), dict(out=h.half())),
            (scan.forward, (x, x), dict(out=turned)), (scan.forward, (x, x), dict(out=h[:1].expand(2, 3, dim))), (scan.step, (x, x, state), {}),
            (scan.step, (x[:, 0], x[:, 0], None), {}), (scan.step, (x[:, 0], x[:, 0], state[:1]), {}), (scan.step, (x[:, 0], x[:, 0], state), dict(out=x)),
            (scan.grad, (x, x, x, h[:1]), {}), (scan.grad, (x.half(), x, x, h), {}), (scan.grad, (x, x, x, h), dict(dz=h)), (scan.grad, (x, x, x, h), dict(dv=turned)),
            (scan.grad, (x, x, x, h), dict(initial=state, d_initial=state)), (scan.grad, (x, x, x, h), dict(d_final=state[:1])), (scan.grad, (x, x, x, h), dict(d_initial=state.double())),
            (drop, (x.cpu(), 1), {}), (drop, (x.double(), 1), {}), (drop, (x, -1), {}), (drop, (x, 2 ** 64), {}), (drop, (x, torch.tensor([1])), {}),
            (drop, (x, torch.tensor([1.0], device="cuda")), {}), (drop, (x, torch.tensor([1, 2], device="cuda")), {}), (drop, (x, 1), dict(residual=x.half(), dtype=F32)),
            (drop, (x, 1), dict(residual=x[:1])), (drop, (x, 1), dict(out=y[:1])), (drop, (x, 1), dict(out=turned)), (drop, (x, 1), dict(out=y, dtype=BF16)),
            (drop, (torch.zeros((), device="cuda"), 1), {}), (drop, (x, 1), dict(out=y[:1].expand(2, 3, dim)))):
        _no(bad, f, *a, **k)
    _no(ea.EA_E_UNSUPPORTED, norm.forward, x.half(), dtype=F32)
    _no(ea.EA_E_UNSUPPORTED, norm.forward, x.half(), dtype=BF16)
    _no(ea.EA_E_UNSUPPORTED, drop, x.half(), 1, dtype=BF16)
    for make in (lambda: ea.LayerNorm(0, 1), lambda: ea.LayerNorm(8, -1), lambda: ea.LayerNorm(8, 1, eps=0.0), lambda: ea.GatedScan(0),
                 lambda: ea.Dropout(1.5), lambda: ea.Dropout(float("nan")), lambda: ea.Dropout(0.1, seed=-1)):
        _no(bad, make)
    _check_forward(*norm.forward(x, w), x, w, None)
    _check_scan(scan.forward(x, x)[0], None, x, x)
