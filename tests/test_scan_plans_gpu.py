"""The recurrence's plans, each with what a call may ask of it: sequences that are walked along (short ones, and wide batches of
longer ones), tiles, clusters, and narrow tiles (few long sequences of few columns).  Checks and tolerances of
tests/test_block_gpu.py."""
import pytest
import torch

import paper_2205_14473_gb300 as ea
from test_block_gpu import BF16, F16, F32, _check_both, _check_scan, _check_scan_grad, _off, _same, _scan_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


# Wide batches on either side of the lengths and sizes from which they are walked along: 269, 337, 405, 606 and 808 16-byte packs to an
# SM of columns that fill their tiles, 303 of columns that fill an eighth and five eighths of them.
@pytest.mark.parametrize("batch,dim", [(320, 1024), (400, 1024), (482, 1024), (720, 1024), (960, 1024), (46_000, 8), (9200, 40)])
@pytest.mark.parametrize("length", [17, 40, 41, 48, 49, 80, 81, 100, 101])
def test_wide_batches(batch, dim, length):
    z, v, dh, first, last = _scan_inputs(batch, length, dim, BF16, seed=20)
    scan = ea.GatedScan(dim)
    h, final, got = _check_both(scan, z, v, dh, first, last)
    again = scan.forward(z, v, initial=first, final=True)
    assert _same(again[0], h) and _same(again[1], final)
    # a sequence's results do not depend on the others, but for how it is cut into pieces
    few = scan.forward(z[:3], v[:3], initial=first[:3], final=True)
    _check_scan(few[0], few[1], z[:3], v[:3], first[:3])


@pytest.mark.parametrize("batch,length,dim", [(2, 40, 1600), (3, 130, 512), (2, 300, 512), (1, 700, 2048), (1, 1100, 64), (2, 9000, 24), (1, 1100, 33)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_states_in_place(batch, length, dim, dtype):
    """The last states into the first ones' memory (and their gradients'), which every CTA of a cluster has read by then."""
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=21)
    scan = ea.GatedScan(dim)
    h, final, got = _check_both(scan, z, v, dh, first, last)
    for _ in range(30):
        s, d = first.clone(), last.clone()
        out, end = scan.forward(z, v, initial=s, final=s)
        assert end is s and _same(s, final) and _same(out, h)
        assert all(_same(p, q) for p, q in zip(scan.grad(dh, z, v, h, initial=first, d_final=d, d_initial=d), got))


# Of 16-byte accesses a cluster takes 128 rows to a CTA and 64 back, in narrow tiles 512 (and 256), of single elements 32.
@pytest.mark.parametrize("batch,dim,rows,dtype,chunks", [(6, 256, 128, BF16, 3), (6, 256, 128, BF16, 5), (6, 256, 64, BF16, 3), (6, 256, 64, BF16, 7),
                                                         (1, 64, 512, F16, 3), (1, 64, 512, F16, 5), (1, 64, 256, F16, 11), (1, 33, 32, F32, 3),
                                                         (1, 33, 32, F32, 6), (1, 33, 32, F32, 9), (1, 33, 32, F32, 13), (1, 33, 32, F32, 15)])
def test_clusters_of_every_number_of_chunks(batch, dim, rows, dtype, chunks):
    """No more CTAs in a cluster than the sequence has chunks, so also numbers that are no powers of two."""
    z, v, dh, first, last = _scan_inputs(batch, chunks * rows - 1, dim, dtype, seed=22)
    scan = ea.GatedScan(dim)
    _check_both(scan, z, v, dh, first, last)
    scan.sync()


# batch, length, dim of each plan, in 16 bits and in 32.
PLANS = {
    "short": (5, 5, 40), "short at its limit": (6, 16, 264), "wide": (320, 45, 1024), "wide and thin": (9200, 70, 40), "tiles": (100, 70, 512),
    "tiles of several chunks": (30, 300, 512), "clusters": (6, 700, 256), "narrow tiles": (4, 1500, 64),
}


def _ends_of(batch, length, kind):
    g = torch.Generator().manual_seed(batch + length)
    ends = torch.randint(0, length + 1, (batch,), generator=g)
    ends[:4] = torch.tensor([0, 1, length, length - 1])
    return ends.to(kind).cuda()


def _halves_of(a, b):
    both = torch.cat([a, b], 2)
    return both[..., :a.shape[2]], both[..., a.shape[2]:]


def _by_time(t):
    return t.transpose(0, 1).contiguous().transpose(0, 1)


def _inside(t, k):
    """A copy of t in longer and more rows, k elements in, and the whole of it."""
    whole = torch.full((t.shape[0], t.shape[1] + 2, t.shape[2] + 16), 7.0, device="cuda", dtype=t.dtype)
    piece = whole[:, 1:-1, k:k + t.shape[2]]
    piece.copy_(t)
    return piece, whole


@pytest.mark.parametrize("layout", ["rows", "halves", "by time", "pieces", "pieces off a boundary", "in place"])
@pytest.mark.parametrize("dtype,kind", [(BF16, torch.int64), (F16, torch.int32), (F32, torch.int32)])
@pytest.mark.parametrize("plan", PLANS)
def test_ragged_batches_of_every_plan(plan, dtype, kind, layout):
    """Lengths of zero, one, all rows and between, NaN behind them, in the layouts that a call takes."""
    batch, length, dim = PLANS[plan]
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=23)
    lengths = _ends_of(batch, length, kind)
    behind = torch.arange(length, device="cuda")[None] >= lengths[:, None]
    clean = [t.masked_fill(behind[..., None], 0.0) for t in (z, v, dh)]
    for t in (z, v, dh):
        t[behind] = float("nan")
    scan, wholes, out, dz, dv = ea.GatedScan(dim), [], None, None, None
    if layout == "halves":
        (z, v), (dz, dv) = _halves_of(z, v), _halves_of(z, v)
    elif layout == "by time":
        z, v, dh, out, dz, dv = (_by_time(t) for t in (z, v, dh, z, z, v))
    elif layout.startswith("pieces"):
        k = 8 if layout == "pieces" else 3
        (z, _), (v, _), (dh, _) = (_inside(t, k) for t in (z, v, dh))
        (out, a), (dz, b), (dv, c) = (_inside(t, k) for t in (z, z, v))
        wholes = [(a, out), (b, dz), (c, dv)]
        first, last = _off(first, k), _off(last, k)
    if layout == "in place":
        out = z.clone()
        h, final = scan.forward(out, v, initial=first, lengths=lengths, out=out, final=True)
    else:
        h, final = scan.forward(z, v, initial=first, lengths=lengths, out=out, final=True)
    assert out is None or h is out
    _check_scan(h, final, clean[0], clean[1], first, lengths)
    assert _same(final[0], first[0])
    h = h.masked_fill(behind[..., None], float("nan"))
    if layout == "in place":
        dz, dv, d = z, dh, last.clone()
        got = scan.grad(dv, dz, v, h, initial=first, lengths=lengths, d_final=d, dz=dz, dv=dv, d_initial=d)
    else:
        got = scan.grad(dh, z, v, h, initial=first, lengths=lengths, d_final=last, dz=dz, dv=dv, d_initial=True)
    _check_scan_grad(got, clean[2], clean[0], clean[1], h.masked_fill(behind[..., None], 0.0), first, lengths, last)
    assert _same(got[2][0], last[0])
    for whole, piece in wholes:  # nothing beside what was asked for
        piece.fill_(7.0)
        assert (whole == 7.0).all()
    scan.sync()


@pytest.mark.parametrize("dtype,kind", [(BF16, torch.int64), (F16, torch.int32)])
@pytest.mark.parametrize("plan", PLANS)
def test_lengths_outside_the_rows_of_every_plan(plan, dtype, kind):
    """They count as the nearest that are inside, and sync() raises for them, once."""
    batch, length, dim = PLANS[plan]
    z, v, dh, first, last = _scan_inputs(batch, length, dim, dtype, seed=24)
    lengths = _ends_of(batch, length, kind)
    inside = lengths.clone()
    lengths[0], lengths[2], lengths[3], inside[3] = -1, length + 1, torch.iinfo(kind).max, length
    scan = ea.GatedScan(dim)
    want = scan.forward(z, v, initial=first, lengths=inside, final=True)
    back = scan.grad(dh, z, v, want[0], initial=first, lengths=inside, d_final=last, d_initial=True)
    scan.sync()
    for f, ref in ((lambda: scan.forward(z, v, initial=first, lengths=lengths, final=True), want),
                   (lambda: scan.grad(dh, z, v, want[0], initial=first, lengths=lengths, d_final=last, d_initial=True), back)):
        assert all(_same(a, b) for a, b in zip(f(), ref))
        with pytest.raises(ea.EAError) as ex:
            scan.sync()
        assert ex.value.status == ea.EA_E_DEVICE_CHECK
        scan.sync()
