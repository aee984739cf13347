"""The recurrence's exchange between the CTAs of a cluster where a wait runs out, without a fault: one CTA of a self-test stops
sending halfway, the others' waits reach a short limit, and the kernel ends with a status that the host reads, no CTA having left
its cluster before the last one has stopped sending."""
import ctypes

import pytest
import torch

import paper_2205_14473_gb300 as ea

LIMIT = 2_000_000  # cycles, about a millisecond


def _exchange(limit, silent):
    out = ctypes.c_int32(-1)
    status = ea.lib().ea_scan_selftest_exchange(limit, silent, torch.cuda.current_stream().cuda_stream, ctypes.byref(out))
    return status, out.value


def test_refusals(ea_lib):
    out = ctypes.c_int32(-1)
    for limit, silent, at in ((0, -1, out), (-1, 0, out), (4_000_000_001, -1, out), (LIMIT, -2, out), (LIMIT, 4, out), (LIMIT, -1, None)):
        assert ea_lib.ea_scan_selftest_exchange(limit, silent, None, at) == ea.EA_E_INVAL and ea_lib.ea_last_error(None)
    assert out.value == -1


@pytest.mark.gpu
def test_waits_that_run_out_end_the_kernel():
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    assert _exchange(200 * LIMIT, -1) == (ea.EA_OK, 0)
    for silent in range(4):
        assert _exchange(LIMIT, silent) == (ea.EA_OK, 1)
    assert _exchange(200 * LIMIT, -1) == (ea.EA_OK, 0)
    # The recurrence in clusters works as before: 40 rows of at most ten roundings each, in either evaluation.
    z, v = torch.randn(2, 2, 5000, 64, device="cuda").unbind()
    scan = ea.GatedScan(64)
    h, _ = scan.forward(z, v)
    state = torch.zeros(2, 64, device="cuda")
    rows = [scan.step(z[:, t], v[:, t], state) for t in range(40)]
    assert (h[:, :40] - torch.stack(rows, 1)).abs().max() <= 800 * 2.0 ** -24 * v.abs().max()
    scan.sync()


@pytest.mark.gpu
@pytest.mark.parametrize("batch,length,dim", [(1, 300, 512), (1, 700, 2048), (2, 5000, 64), (1, 9000, 256), (3, 1200, 33)])
def test_every_run_of_clusters_gives_the_same_bits(batch, length, dim):
    """In clusters of two and more, wide and narrow tiles and single elements: what another CTA of the cluster sends is seen
    whole, every time."""
    assert [_exchange(200_000_000, -1) for _ in range(200)] == [(ea.EA_OK, 0)] * 200
    z, v, dh = torch.randn(3, batch, length, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(length)).unbind()
    scan = ea.GatedScan(dim)
    h, final = scan.forward(z, v, final=True)
    want = [h, final, *scan.grad(dh, z, v, h, d_initial=True)]
    for _ in range(50):
        out, last = scan.forward(z, v, final=True)
        assert all(torch.equal(a, b) for a, b in zip(want, [out, last, *scan.grad(dh, z, v, h, d_initial=True)]))
    scan.sync()
