"""What include/ea_block.h says of the recurrence's gates, and of what their rounding does over many rows."""
import pytest
import torch

import paper_2205_14473_gb300 as ea

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


def _rel(z):
    """Of a gate, relative, in units of 2^-23: 2 of the power of two and 0.61 |z| of its exponent (a product with the rounded log2 e,
    0.5 and 0.11 units of 2^-23 of 1.4427 |z|, times ln 2), which pass on to f or 1 - f at most as they are; 0.5 of the sum 1 + e, 1 of
    the reciprocal, 0.5 of the product e f: 4 + 0.61 |z| together."""
    return (4 + 0.7 * z.abs()) * UNIT


def test_gates_over_their_range():
    """f and 1 - f by themselves: a step from a state of 1 with v = 0, and from 0 with v = 1."""
    dim = 1 << 20
    scan = ea.GatedScan(dim)
    z = torch.linspace(-100, 100, 4 * dim, device="cuda").view(4, dim)
    one, zero = torch.ones_like(z), torch.zeros_like(z)
    for state, v, want in ((one, zero, torch.sigmoid(z.double())), (zero, one, torch.sigmoid(-z.double()))):
        got = scan.step(z, v, state.clone()).double()
        assert ((got - want).abs() <= _rel(z.double()) * want + 2.0 ** -126).all()
