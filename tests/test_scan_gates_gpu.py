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


@pytest.mark.parametrize("length,batch,copies", [(65_536, 1, 1), (65_536, 1, 20), (2000, 3, 8), (90, 2000, 8)])
@pytest.mark.parametrize("v", [1.0, 3.0])
def test_gates_that_nearly_hold(length, batch, copies, v):
    """Constant gates and inputs, from a state of 0 and (v = 3) of 5: every weight of a state and so the state itself, of terms of one
    sign, is off by what its gate's 1 - f is, and by at most 2^-21 a row that it is carried through: the rounding of f (0.5 of the
    sum, 1 of the reciprocal, at z = 0 1 of the power of two) and of the state's sum (0.5), each in units of 2^-23, and as much
    again for pieces that are joined.  dv, of gradients of one sign, the same."""
    gates = torch.tensor([0.0, 2.0, 6.0, 8.0, 10.0, 12.0, 14.0, 16.0, 17.0, 20.0, 40.0, 80.0], device="cuda").repeat(copies)
    dim = gates.numel()
    z = gates.expand(batch, length, dim).contiguous()
    first = 0.0 if v == 1.0 else 5.0
    x, dh = torch.full_like(z, v), torch.ones_like(z)
    scan = ea.GatedScan(dim)
    h, final = scan.forward(z, x, initial=torch.full((batch, dim), first, device="cuda"), final=True)
    g = gates.double()
    # f^n and 1 - f^n of the logarithm of f, each without cancellation
    log_f = -torch.log1p(torch.exp(-g))
    n = torch.arange(1, length + 1, device="cuda", dtype=torch.float64)[:, None]
    new = v * -torch.expm1(n * log_f)
    want = first * torch.exp(n * log_f) + new
    bound = (_rel(g) * new + n * 2.0 ** -21 * want) * 1.05 + 2.0 ** -126 * (1 + n)
    assert ((h.double() - want).abs() <= bound).all()
    assert ((final.double() - want[-1]).abs() <= bound[-1]).all()
    dz, dv, _ = scan.grad(dh, z, x, h)
    # g of row t: the sum of f^k for the rows from there on, (1 - f^m) / (1 - f)
    want = -torch.expm1(n * log_f).flip(0)
    bound = (2 * _rel(g) + n.flip(0) * 2.0 ** -21) * want * 1.05 + 2.0 ** -126 * (1 + n)
    assert ((dv.double() - want).abs() <= bound).all()
