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
