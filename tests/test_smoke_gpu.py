"""What smoke() runs on the device is the package's kernels: the references it checks them against are few operations there."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

pytestmark = pytest.mark.gpu


class _Device(TorchDispatchMode):
    """Counts operations of torch that give a tensor on the device."""

    count = 0

    def __torch_dispatch__(self, f, types, args=(), kwargs=None):
        out = f(*args, **(kwargs or {}))
        self.count += any(isinstance(t, torch.Tensor) and t.is_cuda for t in (out if isinstance(out, (list, tuple)) else (out,)))
        return out


def test_the_block_is_checked_on_the_cpu():
    import __graft_entry__ as G

    G.build()
    torch.cuda.set_device(0)
    with _Device() as seen:
        G.smoke_block()
    assert 0 < seen.count < 60  # inputs, results, one sum; a reference of 70 rows is some hundreds
