"""The operators of include/ea_lm.h without a GPU: what they refuse before any CUDA call, and the sizes of their
workspaces."""
import ctypes
import os
import subprocess

import pytest

import paper_2205_14473_gb300 as ea
from paper_2205_14473_gb300 import lm_abi as A


def _embed(**kw):
    c = dict(vocab=100, dim=8, max_tokens=64, padding=-1, scale=1.0)
    c.update(kw)
    return A.ea_embed_config(*[c[k] for k in ("vocab", "dim", "max_tokens", "padding", "scale")])


def _norm(sizes=(5, 0, 7), n=None, kind=A.EA_T_F32):
    arr = (ctypes.c_int64 * max(len(sizes), 1))(*sizes)
    c = A.ea_grad_norm_config(len(sizes) if n is None else n, kind, ctypes.cast(arr, ctypes.POINTER(ctypes.c_int64)))
    c.keep = arr
    return c


def _adamw(tensor=None, **kw):
    t = dict(size=10, param=4096, m=4096, v=4096, m_scale=4096, v_scale=4096, copy=0, weight_decay=0.1, lr_scale=1.0)
    t.update(tensor or {})
    c = dict(n_tensors=1, param_type=A.EA_T_F32, grad_type=A.EA_T_F32, copy_type=A.EA_T_BF16, state_bits=32, beta1=0.9,
             beta2=0.999, eps=1e-8, seed=0, step=0)
    c.update(kw)
    arr = (A.ea_adamw_tensor * 1)(A.ea_adamw_tensor(*[t[f] for f, _ in A.ea_adamw_tensor._fields_]))
    out = A.ea_adamw_config(*[c[f] for f, _ in A.ea_adamw_config._fields_[:-1]],
                            ctypes.cast(arr, ctypes.POINTER(A.ea_adamw_tensor)))
    out.keep = arr
    return out


def _refused(L, kind, config, status):
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    assert getattr(L, kind + "_workspace_bytes")(config, ctypes.byref(n)) == status
    assert L.ea_last_error(None)
    assert getattr(L, kind + "_init")(config, 4096, 1 << 30, None, ctypes.byref(h)) == status
    assert not h.value


@pytest.mark.parametrize("bad", [dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(dim=0), dict(dim=2 ** 24 + 1),
                                 dict(max_tokens=-1), dict(max_tokens=2 ** 30 + 1), dict(padding=-2), dict(padding=100),
                                 dict(scale=float("nan")), dict(scale=float("inf"))])
def test_embedding_refusals(ea_lib, bad):
    _refused(ea_lib, "ea_embed", _embed(**bad), ea.EA_E_INVAL)


@pytest.mark.parametrize("bad", [dict(sizes=()), dict(sizes=(3, -1)), dict(kind=A.EA_T_I32), dict(n=2 ** 20 + 1),
                                 dict(sizes=(2 ** 40 + 1,))])
def test_norm_refusals(ea_lib, bad):
    _refused(ea_lib, "ea_grad_norm", _norm(**bad), ea.EA_E_INVAL)


@pytest.mark.parametrize("status,tensor,bad", [
    (ea.EA_E_INVAL, {}, dict(n_tensors=0)), (ea.EA_E_INVAL, {}, dict(state_bits=16)),
    (ea.EA_E_INVAL, {}, dict(beta1=1.0)), (ea.EA_E_INVAL, {}, dict(beta2=-0.1)), (ea.EA_E_INVAL, {}, dict(eps=0.0)),
    (ea.EA_E_INVAL, {}, dict(step=-1)), (ea.EA_E_INVAL, {}, dict(step=2 ** 32)), (ea.EA_E_INVAL, {}, dict(grad_type=9)),
    (ea.EA_E_UNSUPPORTED, {}, dict(param_type=A.EA_T_F16)), (ea.EA_E_INVAL, dict(size=-1), {}),
    (ea.EA_E_INVAL, dict(param=0), {}), (ea.EA_E_ALIGN, dict(param=4098), {}), (ea.EA_E_ALIGN, dict(m=4097), {}),
    (ea.EA_E_INVAL, dict(weight_decay=-1.0), {}), (ea.EA_E_INVAL, dict(weight_decay=float("nan")), {}),
    (ea.EA_E_INVAL, dict(lr_scale=-1.0), {}), (ea.EA_E_INVAL, dict(v=0), dict(state_bits=8)),
    (ea.EA_E_INVAL, dict(m_scale=0), dict(state_bits=8)), (ea.EA_E_ALIGN, dict(v_scale=4098), dict(state_bits=8)),
    (ea.EA_E_INVAL, dict(copy=4096), dict(copy_type=A.EA_T_F32)), (ea.EA_E_ALIGN, dict(copy=4097), {}),
])
def test_adamw_refusals(ea_lib, status, tensor, bad):
    _refused(ea_lib, "ea_adamw", _adamw(tensor, **bad), status)


@pytest.mark.parametrize("kind,config", [("ea_embed", _embed()), ("ea_grad_norm", _norm()), ("ea_adamw", _adamw())])
def test_workspace_checks_come_before_the_device(ea_lib, kind, config):
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    assert getattr(ea_lib, kind + "_workspace_bytes")(config, ctypes.byref(n)) == ea.EA_OK and n.value >= 256
    init = getattr(ea_lib, kind + "_init")
    for ws, size in ((None, n.value), (4096 + 16, n.value), (4096, n.value - 1)):
        assert init(config, ws, size, None, ctypes.byref(h)) == ea.EA_E_WORKSPACE
    assert init(config, 4096, n.value, None, None) == ea.EA_E_INVAL
    assert getattr(ea_lib, kind + "_workspace_bytes")(config, None) == ea.EA_E_INVAL
    assert getattr(ea_lib, kind + "_workspace_bytes")(None, ctypes.byref(n)) == ea.EA_E_INVAL
    assert getattr(ea_lib, kind + "_destroy")(None) == ea.EA_OK


def test_null_handles(ea_lib):
    one = (ctypes.c_void_p * 1)(4096)
    call = A.ea_embed_call(1, 1, 1, 1, 8, 8, 8, A.EA_T_I64, A.EA_T_F32, A.EA_T_F32)
    assert ea_lib.ea_embed_lookup(None, call, 4096, 4096, 4096) == ea.EA_E_INVAL
    assert ea_lib.ea_embed_grad(None, call, 4096, 4096, 4096, 0) == ea.EA_E_INVAL
    assert ea_lib.ea_embed_sync_status(None) == ea.EA_E_INVAL
    assert ea_lib.ea_grad_norm(None, one, 1.0, 1.0, 4096) == ea.EA_E_INVAL
    assert ea_lib.ea_adamw_step(None, one, 1e-3, None) == ea.EA_E_INVAL
    assert ea_lib.ea_adamw_step_index(None, None) == ea.EA_E_INVAL


def test_init_without_a_device(tmp_path):
    """Where the device cannot be asked for its SMs an init call ends there: built with the C++ library's assertions, it
    reports the CUDA error instead of sharing work out over no SMs."""
    from paper_2205_14473_gb300 import build as B

    main = tmp_path / "main.cpp"
    main.write_text("""
        #include "ea_lm.h"
        namespace ea { void set_last_error(const char *) {} }
        int main()
        {
            const int64_t size = 10;
            void *at = reinterpret_cast<void *>(4096);
            ea_grad_norm_config n{1, EA_T_F32, &size};
            ea_norm *norm = nullptr;
            ea_adamw_tensor t{size, at, at, at, nullptr, nullptr, nullptr, 0.0f, 1.0f};
            ea_adamw_config a{1, EA_T_F32, EA_T_F32, EA_T_BF16, 32, 0.9f, 0.999f, 1e-8f, 0, 0, &t};
            ea_adamw *adamw = nullptr;
            if (ea_grad_norm_init(&n, at, size_t{1} << 20, nullptr, &norm) != EA_E_CUDA || norm) return 1;
            if (ea_adamw_init(&a, at, size_t{1} << 20, nullptr, &adamw) != EA_E_CUDA || adamw) return 2;
            return 0;
        }""")
    units = [os.path.join(B.CSRC, f) for f in ("ea_norm.cu", "ea_adamw.cu")]
    subprocess.run([B.NVCC, "-gencode", "arch=compute_103a,code=compute_103a", "-std=c++17", "--threads", "2", "-Xcompiler",
                    "-D_GLIBCXX_ASSERTIONS", "-I" + os.path.join(B.ROOT, "include"), "-o", tmp_path / "main", main, *units], check=True)
    assert subprocess.run([tmp_path / "main"], env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}).returncode == 0


@pytest.mark.parametrize("here,raw", [(0, 7), (1, 7), (1, 5)])
def test_calls_run_on_the_handles_device(monkeypatch, here, raw):
    """A handle of device 1 on stream 7, called while device `here` and stream `raw` of device 1 are current (all of it
    faked): the library sees device 1, the streams wait for one another where they differ, and device `here` is current
    again afterwards."""
    import contextlib
    from types import SimpleNamespace

    import torch

    from paper_2205_14473_gb300 import lm

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
        names = ("ea_embed_lookup", "ea_embed_grad", "ea_embed_sync_status", "ea_grad_norm", "ea_adamw_step", "ea_adamw_step_index",
                 "ea_embed_destroy", "ea_grad_norm_destroy", "ea_adamw_destroy")
        h.__dict__.update(device=torch.device("cpu"), _index=1, _raw=7, stream=stream(7), h=1, _L=SimpleNamespace(**{n: call(n) for n in names}),
                          **fields)
        return h

    def seen(name, tensors, f):
        log.clear()
        f()
        want = [(name, 1)] if raw == 7 else [(7, 5), (name, 1), (5, 7)] + [("record", 7)] * tensors
        assert log == want and device[0] == here, name

    w, g = torch.ones(4, 2), torch.ones(8)
    table = handle(lm.Embedding, vocab=4, dim=2, _shape=torch.Size((4, 2)), _c=A.ea_embed_call())
    ids = torch.tensor([1, 3])
    seen("ea_embed_lookup", 3, lambda: table.lookup(ids, w))
    seen("ea_embed_grad", 3, lambda: table.grad(ids, torch.ones(2, 2)))
    norm = handle(lm.GradNorm, sizes=[8], dtype=torch.float32)
    seen("ea_grad_norm", 2, lambda: norm([g]))
    opt = handle(lm.AdamW, sizes=[8], dtype=torch.float32, _touched=(g, g, g), _modified=(g,))
    seen("ea_adamw_step", 5, lambda: opt.step([g], lr=1e-3, clip=torch.ones(2)))
    log.clear()
    table.sync()
    assert opt.t == 0 and log == [("ea_embed_sync_status", 1), ("ea_adamw_step_index", 1)] and device[0] == here


def test_refusals_of_what_is_not_a_cuda_tensor(ea_lib):
    """Host tensors and things that are no tensors are refused as every other argument is, by EAError."""
    import torch

    p = torch.zeros(3)
    for f in (lambda: ea.AdamW([p]), lambda: ea.AdamW([p], state_bits=8), lambda: ea.AdamW([1.0]), lambda: ea.AdamW([p, None]),
              lambda: ea.TensorList([None]), lambda: ea.TensorList(["a", p]), lambda: ea.GradNorm([3], device="cpu"),
              lambda: ea.Embedding(3, 4, 5, device="cpu"), lambda: ea.AdamW([p], copies=[1.0]),
              lambda: ea.AdamW([p], states={"m": [1.0], "v": [1.0]})):
        with pytest.raises(ea.EAError) as ex:
            f()
        assert ex.value.status == ea.EA_E_INVAL and str(ex.value)


def test_selftest_refuses_null(ea_lib):
    assert ea_lib.ea_adamw_selftest_sqrt(None, None) == ea.EA_E_INVAL


@pytest.mark.parametrize("kind,config,edge,past", [
    ("ea_embed", _embed, dict(vocab=2 ** 31 - 2), dict(vocab=2 ** 31 - 1)), ("ea_embed", _embed, dict(dim=2 ** 20), dict(dim=2 ** 20 + 1)),
    ("ea_embed", _embed, dict(max_tokens=2 ** 30), dict(max_tokens=2 ** 30 + 1)), ("ea_embed", _embed, dict(max_tokens=0), dict(max_tokens=-1)),
    ("ea_embed", _embed, dict(padding=99), dict(padding=100)), ("ea_embed", _embed, dict(padding=-1), dict(padding=-2)),
    ("ea_grad_norm", _norm, dict(sizes=(2 ** 40,)), dict(sizes=(2 ** 40 + 1,))),
    ("ea_grad_norm", _norm, dict(sizes=(0,) * 2 ** 20), dict(sizes=(0,) * (2 ** 20 + 1))),
    ("ea_adamw", _adamw, dict(tensor=dict(size=2 ** 40)), dict(tensor=dict(size=2 ** 40 + 1))),
    ("ea_adamw", _adamw, dict(beta1=0.0), dict(beta1=-1e-45)), ("ea_adamw", _adamw, dict(eps=1.1e-30), dict(eps=0.9e-30)),
    ("ea_adamw", _adamw, dict(step=2 ** 32 - 1), dict(step=2 ** 32)), ("ea_adamw", _adamw, dict(beta2=1 - 2.0 ** -24), dict(beta2=1.0)),
])
def test_limits_on_both_sides(ea_lib, kind, config, edge, past):
    n, query = ctypes.c_size_t(0), getattr(ea_lib, kind + "_workspace_bytes")
    assert query(config(**edge), ctypes.byref(n)) == ea.EA_OK and n.value >= 256
    assert query(config(**past), ctypes.byref(n)) == ea.EA_E_INVAL
