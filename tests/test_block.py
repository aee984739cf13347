"""The operators of include/ea_block.h without a GPU: what they refuse before any CUDA call, and the sizes of their
workspaces."""
import ctypes

import pytest

import paper_2205_14473_gb300 as ea
from paper_2205_14473_gb300 import block_abi as A
from paper_2205_14473_gb300 import lm_abi as T


def _norm(dim=8, max_rows=64, eps=1e-5):
    return A.ea_layernorm_config(dim, max_rows, eps)


def _scan(dim=8):
    return A.ea_scan_config(dim)


def _drop(p=0.1, seed=0):
    return A.ea_dropout_config(p, seed)


KINDS = {"ea_layernorm": _norm, "ea_scan": _scan, "ea_dropout": _drop}


@pytest.mark.parametrize("kind,bad", [
    ("ea_layernorm", dict(dim=0)), ("ea_layernorm", dict(dim=2 ** 20 + 1)), ("ea_layernorm", dict(max_rows=-1)),
    ("ea_layernorm", dict(max_rows=2 ** 30 + 1)), ("ea_layernorm", dict(eps=0.0)), ("ea_layernorm", dict(eps=-1.0)),
    ("ea_layernorm", dict(eps=float("nan"))), ("ea_layernorm", dict(eps=float("inf"))),
    ("ea_scan", dict(dim=0)), ("ea_scan", dict(dim=-5)), ("ea_scan", dict(dim=2 ** 20 + 1)),
    ("ea_dropout", dict(p=-0.1)), ("ea_dropout", dict(p=1.0000001)), ("ea_dropout", dict(p=float("nan"))),
])
def test_refusals(ea_lib, kind, bad):
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    assert getattr(ea_lib, kind + "_workspace_bytes")(KINDS[kind](**bad), ctypes.byref(n)) == ea.EA_E_INVAL
    assert ea_lib.ea_last_error(None)
    assert getattr(ea_lib, kind + "_init")(KINDS[kind](**bad), 4096, 1 << 30, None, ctypes.byref(h)) == ea.EA_E_INVAL
    assert not h.value


@pytest.mark.parametrize("kind,edge", [
    ("ea_layernorm", dict(dim=1, max_rows=0)), ("ea_layernorm", dict(dim=2 ** 20, max_rows=2 ** 30)), ("ea_layernorm", dict(eps=1.1e-30)),
    ("ea_scan", dict(dim=1)), ("ea_scan", dict(dim=2 ** 20)), ("ea_dropout", dict(p=0.0)), ("ea_dropout", dict(p=1.0)),
    ("ea_dropout", dict(seed=2 ** 64 - 1)),
])
def test_limits(ea_lib, kind, edge):
    n = ctypes.c_size_t(0)
    assert getattr(ea_lib, kind + "_workspace_bytes")(KINDS[kind](**edge), ctypes.byref(n)) == ea.EA_OK
    assert n.value < 64 << 20


@pytest.mark.parametrize("kind", KINDS)
def test_arguments_come_before_the_device(ea_lib, kind):
    config, n, h = KINDS[kind](), ctypes.c_size_t(0), ctypes.c_void_p()
    size, init = getattr(ea_lib, kind + "_workspace_bytes"), getattr(ea_lib, kind + "_init")
    assert size(config, ctypes.byref(n)) == ea.EA_OK
    for ws, have in ((None, n.value), (4096 + 16, n.value), (4096, n.value - 1)):
        if n.value:
            assert init(config, ws, have, None, ctypes.byref(h)) == ea.EA_E_WORKSPACE
    assert init(config, 4096, n.value, None, None) == ea.EA_E_INVAL
    assert init(None, 4096, n.value, None, ctypes.byref(h)) == ea.EA_E_INVAL
    assert size(config, None) == ea.EA_E_INVAL
    assert size(None, ctypes.byref(n)) == ea.EA_E_INVAL
    assert getattr(ea_lib, kind + "_destroy")(None) == ea.EA_OK


def test_init_without_a_device(ea_lib):
    """Where there is no device to ask, an init call reports the CUDA error and makes no handle."""
    import torch

    if torch.cuda.is_available():
        pytest.skip("there is a device")
    for kind, config in KINDS.items():
        h = ctypes.c_void_p()
        assert getattr(ea_lib, kind + "_init")(config(), 4096, 1 << 30, None, ctypes.byref(h)) == ea.EA_E_CUDA and not h.value


def test_null_handles(ea_lib):
    assert ea_lib.ea_layernorm_forward(None, A.ea_layernorm_call(), 4096, None, None, 4096, None) == ea.EA_E_INVAL
    assert ea_lib.ea_layernorm_backward(None, A.ea_layernorm_call(), 4096, 4096, 4096, None, None, 4096, None, None, 0) == ea.EA_E_INVAL
    assert ea_lib.ea_scan_forward(None, A.ea_scan_call(), 4096, 4096, None, None, 4096, None) == ea.EA_E_INVAL
    assert ea_lib.ea_scan_backward(None, A.ea_scan_call(), 4096, 4096, 4096, 4096, None, None, None, 4096, 4096, None) == ea.EA_E_INVAL
    assert ea_lib.ea_scan_sync_status(None) == ea.EA_E_INVAL
    assert ea_lib.ea_dropout_apply(None, A.ea_dropout_call(), 4096, None, 0, None, 4096) == ea.EA_E_INVAL


def test_refusals_of_what_is_not_a_cuda_tensor(ea_lib):
    for f in (lambda: ea.LayerNorm(8, 4, device="cpu"), lambda: ea.GatedScan(8, device="cpu"), lambda: ea.Dropout(0.1, device="cpu"),
              lambda: ea.Dropout(0.1, seed=-1, device="cpu"), lambda: ea.Dropout(0.1, seed=2 ** 64, device="cpu")):
        with pytest.raises(ea.EAError) as ex:
            f()
        assert ex.value.status == ea.EA_E_INVAL and str(ex.value)


def test_types_are_those_of_the_other_header():
    assert (T.EA_T_F32, T.EA_T_BF16, T.EA_T_F16, T.EA_T_I32, T.EA_T_I64) == (0, 1, 2, 3, 4)
    assert ctypes.sizeof(A.ea_layernorm_call) == 96 and ctypes.sizeof(A.ea_scan_call) == 120 and ctypes.sizeof(A.ea_dropout_call) == 80


@pytest.mark.parametrize("here,raw", [(0, 7), (1, 7), (1, 5)])
def test_calls_run_on_the_handles_device(monkeypatch, here, raw):
    """A handle of device 1 on stream 7, called while device `here` and stream `raw` of device 1 are current (all of it
    faked): the library sees device 1, the streams wait for one another where they differ, every tensor that a call touches is
    recorded on the handle's stream, and device `here` is current again afterwards."""
    import contextlib
    from types import SimpleNamespace

    import torch

    from paper_2205_14473_gb300 import block

    log, device = [], [here]

    @contextlib.contextmanager
    def switch(index):
        before, device[0] = device[0], index
        yield
        device[0] = before

    def stream(which):
        return SimpleNamespace(cuda_stream=which, wait_stream=lambda other: log.append((which, other.cuda_stream)))

    def call(name):
        def f(*args):
            log.append((name, device[0]))
            return ea.EA_OK
        return f

    monkeypatch.setattr(torch.cuda, "device", switch)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: stream(raw))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: device[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: raw, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", s.cuda_stream)))

    def handle(kind, **fields):
        h = kind.__new__(kind)
        h.__dict__.update(device=torch.device("cpu"), _index=1, _raw=7, stream=stream(7), h=1,
                          _L=SimpleNamespace(**{n: call(n) for n in A.EXPORTED}), **fields)
        return h

    def seen(name, tensors, f):
        log.clear()
        f()
        want = [(name, 1)] if raw == 7 else [(7, 5), (name, 1), (5, 7)] + [("record", 7)] * tensors
        assert log == want and device[0] == here, name

    norm = handle(block.LayerNorm, dim=4, _row=torch.Size((4,)), _c=A.ea_layernorm_call(), _flat=A.ea_layernorm_call())
    x, w, stats = torch.ones(3, 4), torch.ones(4), torch.ones(3, 2)
    seen("ea_layernorm_forward", 5, lambda: norm.forward(x, w, w))
    seen("ea_layernorm_backward", 8, lambda: norm.grad(x, x, stats, w, add=x, dw=True, db=True))
    scan, z, state = handle(block.GatedScan, dim=4, _c=A.ea_scan_call()), torch.ones(2, 3, 4), torch.ones(2, 4)
    seen("ea_scan_forward", 6, lambda: scan.forward(z, z, initial=state, lengths=torch.tensor([1, 2]), final=True))
    seen("ea_scan_forward", 4, lambda: scan.step(z[:, 0], z[:, 0], state))
    seen("ea_scan_backward", 10, lambda: scan.grad(z, z, z, z, initial=state, lengths=torch.tensor([1, 2]), d_final=state, d_initial=True))
    drop = handle(block.Dropout, _c=A.ea_dropout_call(), _flat=A.ea_dropout_call())
    seen("ea_dropout_apply", 4, lambda: drop(x, torch.tensor([5]), residual=x))
    log.clear()
    scan.sync()
    assert log == [("ea_scan_sync_status", 1)] and device[0] == here
