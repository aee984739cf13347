"""The operators at the two ends of a language-model worker's training step (include/ea_lm.h): embedding
lookup and the table's gradient, the clipped gradient norm, and AdamW over many tensors.

    table = Embedding(vocab, dim, max_tokens, scale=dim ** 0.5)
    y = table.lookup(tokens, weight, dtype=torch.bfloat16)
    ...                                                  # the model, and its gradients
    table.grad(tokens, dy, out=dw)                       # dw may be a piece of a worker's flat gradient
    norm = GradNorm([g.numel() for g in grads])
    opt = AdamW(params, state_bits=8)
    opt.step(grads, lr=1e-3, clip=norm(grads, max_norm=1.0))

As with EARound, the calls only marshal arguments, a handle is bound to one stream (by default the current one
where it is made), and every call is asynchronous on it.  A call made while another stream of the handle's device is
current is ordered after the work of that stream so far, and that stream's later work after the call; which device is
current does not matter.

None of them is an autograd operation: a result has no graph, whether or not an input requires a gradient (Embedding.grad
is lookup's backward pass, for the caller to run).  A tensor that a call writes to counts as modified in place, so a
backward pass that had saved it fails instead of using the new values.
"""
from __future__ import annotations

import ctypes
from itertools import chain

import torch

from . import EA_E_INVAL, EAError, _check, lib
from .lm_abi import (EA_ADAMW_BLOCK, EA_T_BF16, EA_T_F16, EA_T_F32, EA_T_I32, EA_T_I64, _i64, _P,
                     ea_adamw_config, ea_adamw_tensor, ea_embed_call, ea_embed_config, ea_grad_norm_config)

_TYPE = {torch.float32: EA_T_F32, torch.bfloat16: EA_T_BF16, torch.float16: EA_T_F16}
_TOKEN = {torch.int32: EA_T_I32, torch.int64: EA_T_I64}
_C = torch._C


def _refuse(msg: str, status: int = EA_E_INVAL):
    raise EAError(status, msg)


def _need_cuda(device) -> None:
    if device.type != "cuda":
        _refuse(f"the device is {device}: these operators run on CUDA devices")


class _Handle:
    """A library handle with its workspace, on one stream of one device."""

    _kind = ""
    _only = False  # whether there is no other device, which need not be looked at then

    def _open(self, config, stream, device) -> None:
        self.device = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        _need_cuda(self.device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._raw = self.stream.cuda_stream
        self._index = self.device.index
        self._only = torch.cuda.device_count() == 1
        self._L = lib()
        n, h = ctypes.c_size_t(0), _P()
        _check(getattr(self._L, self._kind + "_workspace_bytes")(ctypes.byref(config), ctypes.byref(n)))
        self.workspace_bytes = n.value
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            self.workspace = torch.empty(max(n.value, 256), dtype=torch.uint8, device=self.device)
            _check(getattr(self._L, self._kind + "_init")(ctypes.byref(config), self.workspace.data_ptr(), n.value,
                                                          self._raw, ctypes.byref(h)))
        self.h = h.value

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            getattr(self._L, self._kind + "_destroy")(h)
            self.h = None

    def _call(self, f, args, *tensors) -> None:
        """f, a call of the library on this handle that reads or writes `tensors` (lists of them)."""
        if (self._only or _C._cuda_getDevice() == self._index) and _C._cuda_getCurrentRawStream(self._index) == self._raw:
            status = f(self.h, *args)
        else:
            status = self._call_from_elsewhere(f, args, chain(*tensors))
        if status:
            _check(status)

    def _call_from_elsewhere(self, f, args, tensors) -> int:
        """The same with the handle's device current, and in order with the current stream."""
        with torch.cuda.device(self._index):
            now = torch.cuda.current_stream()
            if now.cuda_stream == self._raw:
                return f(self.h, *args)
            self.stream.wait_stream(now)
            status = f(self.h, *args)
            now.wait_stream(self.stream)
            for t in tensors:
                t.record_stream(self.stream)
            return status

    def _on_device(self, t, what: str) -> None:
        if not isinstance(t, torch.Tensor):
            _refuse(f"{what} is not a tensor")
        if t.device != self.device:
            _refuse(f"{what} is on {t.device}, the handle on {self.device}")


class Embedding(_Handle):
    """A vocab x dim embedding table's lookup and gradient for up to max_tokens tokens a call.

    Both are multiplied by `scale`; `padding_idx` names a token that takes no gradient (its row is looked up
    as any other).  Tables, rows and gradients are float32, bfloat16 or float16, tokens int32 or int64.  A
    token outside [0, vocab) gives a row of zeros and no gradient, and sync() raises for it."""

    _kind = "ea_embed"

    def __init__(self, vocab: int, dim: int, max_tokens: int, scale: float = 1.0, padding_idx=None, stream=None,
                 device=None):
        self.vocab, self.dim, self.max_tokens = int(vocab), int(dim), int(max_tokens)
        padding = -1 if padding_idx is None else int(padding_idx)
        if padding_idx is not None and padding < 0:
            _refuse("padding_idx must be a token or None")
        self._c, self._shape = ea_embed_call(), torch.Size((self.vocab, self.dim))
        self._open(ea_embed_config(self.vocab, self.dim, self.max_tokens, padding, scale), stream, device)

    # What a call has to check goes into the one ea_embed_call of the handle.

    def _tokens(self, tokens):
        """Describes the tokens; returns those to pass: of a layout that two strides do not describe, a copy."""
        c = self._c
        if not isinstance(tokens, torch.Tensor) or tokens.device != self.device:
            self._on_device(tokens, "tokens")
        kind = _TOKEN.get(tokens.dtype)
        if kind is None:
            _refuse(f"tokens are int32 or int64, not {tokens.dtype}")
        c.token_type = kind
        shape = tokens.shape
        if len(shape) == 2:
            c.outer, c.inner = shape
            c.token_outer, c.token_inner = tokens.stride()
        elif len(shape) == 1:
            c.outer, c.inner, c.token_outer, c.token_inner = 1, shape[0], 0, tokens.stride(0)
        else:
            tokens = tokens.contiguous()
            c.outer, c.inner, c.token_outer, c.token_inner = 1, tokens.numel(), 0, 1
        return tokens

    def _rows(self, rows, tokens, name) -> None:
        """Describes the rows that belong to tokens' shape."""
        c = self._c
        if not isinstance(rows, torch.Tensor) or rows.device != self.device:
            self._on_device(rows, name)
        if rows.shape != (*tokens.shape, self.dim):
            _refuse(f"{name} is {tuple(rows.shape)}, not {(*tokens.shape, self.dim)}")
        n = tokens.dim()
        if self.dim > 1 and rows.stride(-1) != 1 or n not in (1, 2) and not rows.is_contiguous():
            _refuse(f"the rows of {name} are not contiguous")
        if n == 2:
            c.row_outer, c.row_inner = rows.stride()[:2]
        else:
            c.row_outer, c.row_inner = 0, rows.stride(0) if n == 1 else self.dim
        self._row_type(rows.dtype, name)

    def _row_type(self, dtype, name) -> None:
        kind = _TYPE.get(dtype)
        if kind is None:
            _refuse(f"{name} is float32, bfloat16 or float16, not {dtype}")
        self._c.row_type = kind

    def _table(self, table, name) -> None:
        c = self._c
        if not isinstance(table, torch.Tensor) or table.device != self.device:
            self._on_device(table, name)
        if table.shape != self._shape:
            _refuse(f"{name} is {tuple(table.shape)}, not {(self.vocab, self.dim)}")
        kind = _TYPE.get(table.dtype)
        if kind is None:
            _refuse(f"{name} is float32, bfloat16 or float16, not {table.dtype}")
        outer, inner = table.stride()
        if inner != 1 and self.dim > 1:
            _refuse(f"the rows of {name} are not contiguous")
        c.table_type, c.table_stride = kind, outer if self.vocab > 1 else max(outer, self.dim)

    def lookup(self, tokens, weight, out=None, dtype=None):
        """scale * weight[tokens], of shape tokens.shape + (dim,), in `dtype` (default: weight's) or into `out`."""
        ids, given = self._tokens(tokens), out is not None
        self._table(weight, "weight")
        if not given:
            out = torch.empty((*tokens.shape, self.dim), dtype=dtype or weight.dtype, device=self.device)
            self._c.row_outer, self._c.row_inner = self._c.inner * self.dim, self.dim
            self._row_type(out.dtype, "out")
        else:
            self._rows(out, tokens, "out")
            if dtype is not None and out.dtype != dtype:
                _refuse(f"out is {out.dtype}, not {dtype}")
        self._call(self._L.ea_embed_lookup, (self._c, ids.data_ptr(), weight.data_ptr(), out.data_ptr()), (ids, weight, out))
        if given:
            _C._increment_version((out,))
        return out

    def grad(self, tokens, dy, out=None, accumulate: bool = False, dtype=torch.float32):
        """The gradient of weight, of shape (vocab, dim), from dy = the gradient of lookup's result, into `out`
        or, with accumulate, added to it."""
        ids, given = self._tokens(tokens), out is not None
        if not given:
            if accumulate:
                _refuse("accumulate needs out")
            out = torch.empty(self._shape, dtype=dtype, device=self.device)
        self._table(out, "out")
        if isinstance(dy, torch.Tensor) and dy.dim() and (dy.stride(-1) != 1 or tokens.dim() not in (1, 2)):
            dy = dy.contiguous()
        self._rows(dy, tokens, "dy")
        self._call(self._L.ea_embed_grad, (self._c, ids.data_ptr(), dy.data_ptr(), out.data_ptr(), int(accumulate)), (ids, dy, out))
        if given:
            _C._increment_version((out,))
        return out

    def sync(self) -> None:
        with torch.cuda.device(self._index):
            _check(self._L.ea_embed_sync_status(self.h))


class TensorList:
    """Contiguous tensors of one type and device, checked once: what step() and GradNorm take in place of a list
    where the same buffers are used every step.  Holds on to the tensors."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        if not self.tensors:
            _refuse("no tensors")
        first = self.tensors[0]
        for i, t in enumerate(self.tensors):
            if not isinstance(t, torch.Tensor):
                _refuse(f"tensor {i} is a {type(t).__name__}")
            if t.dtype != first.dtype or t.device != first.device or not t.is_contiguous():
                _refuse(f"tensor {i} is not a contiguous tensor of {first.dtype} on {first.device}")
        self.dtype, self.device = first.dtype, first.device
        self.sizes = [t.numel() for t in self.tensors]
        self._ptrs = (_P * len(self.tensors))(*[t.data_ptr() for t in self.tensors])


def _grad_list(h, grads) -> TensorList:
    g = grads if type(grads) is TensorList else TensorList(grads)
    if g.device != h.device:
        _refuse(f"the gradients are on {g.device}, the handle on {h.device}")
    if g.dtype != h.dtype:
        _refuse(f"the gradients are {g.dtype}, the handle takes {h.dtype}")
    if g.sizes != h.sizes:
        _refuse("the gradients' sizes are not the handle's")
    return g


class GradNorm(_Handle):
    """The 2-norm of gradients of the given sizes, and the factor that clips them."""

    _kind = "ea_grad_norm"

    def __init__(self, sizes, dtype=torch.float32, stream=None, device=None):
        self.sizes, self.dtype = [int(n) for n in sizes], dtype
        if dtype not in _TYPE:
            _refuse(f"gradients are float32, bfloat16 or float16, not {dtype}")
        arr = (_i64 * len(self.sizes))(*self.sizes)
        self._open(ea_grad_norm_config(len(self.sizes), _TYPE[dtype], ctypes.cast(arr, ctypes.POINTER(_i64))), stream, device)

    def __call__(self, grads, max_norm: float = float("inf"), grad_scale: float = 1.0, out=None):
        """A float32 tensor of two: the norm N of grad_scale * grads, and grad_scale * min(1, max_norm / N), NaN where
        N is not finite.  AdamW.step takes it as `clip`."""
        g, given = _grad_list(self, grads), out is not None
        if not given:
            out = torch.empty(2, dtype=torch.float32, device=self.device)
        else:
            self._on_device(out, "out")
            if out.dtype != torch.float32 or out.numel() != 2 or not out.is_contiguous():
                _refuse("out is two contiguous float32 values")
        self._call(self._L.ea_grad_norm, (g._ptrs, grad_scale, max_norm, out.data_ptr()), (out,), g.tensors)
        if given:
            _C._increment_version((out,))
        return out


class AdamW(_Handle):
    """AdamW over a list of contiguous tensors (float32 or bfloat16), with states in 32 or 8 bits.

    weight_decay and lr_scale are one value or one per tensor.  copies: None, or per tensor None or a bfloat16 /
    float16 tensor that receives the new parameters too (the model's copy of float32 parameters).  states: None
    (zeros are made) or a dict of lists of contiguous tensors, one per parameter: "m" and "v" (float32) for 32
    bits; "m" and "r" (float8_e4m3fn, r the root of the second moment) with "m_scale" and "r_scale" (float32, one
    value per 256 coordinates) for 8.  step: the steps that these states have behind them.  seed: key of the
    8-bit states' stochastic rounding.  self.states holds the states' tensors, self.t the steps taken."""

    _kind = "ea_adamw"

    def __init__(self, params, state_bits: int = 32, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01,
                 lr_scale=1.0, grad_dtype=None, copies=None, states=None, seed: int = 0, step: int = 0, stream=None):
        self.params = TensorList(params)
        n = len(self.params.tensors)
        self.sizes, self.param_dtype = self.params.sizes, self.params.dtype
        self.dtype = grad_dtype or self.param_dtype
        if self.param_dtype not in _TYPE or self.dtype not in _TYPE:
            _refuse(f"parameters and gradients are float32, bfloat16 or float16, not {self.param_dtype} and {self.dtype}")
        device = self.params.device
        _need_cuda(device)
        names = {32: ("m", "v"), 8: ("m", "r", "m_scale", "r_scale")}.get(state_bits)
        if names is None:
            _refuse("state_bits is 32 or 8")
        lengths = {k: [-(-s // EA_ADAMW_BLOCK) for s in self.sizes] if k.endswith("_scale") else self.sizes for k in names}
        dtypes = {k: torch.float8_e4m3fn if state_bits == 8 and not k.endswith("_scale") else torch.float32 for k in names}
        if states is None:
            with torch.cuda.device(device), torch.cuda.stream(stream or torch.cuda.current_stream(device)):
                states = {k: list(torch.zeros(sum(lengths[k]), device=device, dtype=dtypes[k]).split(lengths[k]))
                          for k in names}
        if set(states) != set(names):
            _refuse(f"states are {', '.join(names)}, not {', '.join(states)}")
        self.states = {k: list(v) for k, v in states.items()}
        for k in names:
            for i, t in enumerate(self.states[k]):
                if not isinstance(t, torch.Tensor) or t.dtype != dtypes[k] or t.device != device or not t.is_contiguous():
                    _refuse(f"{k}[{i}] is not a contiguous tensor of {dtypes[k]} on {device}")
            if [t.numel() for t in self.states[k]] != lengths[k]:
                _refuse(f"{k} does not have the sizes of the parameters' states")
        self.copies = [None] * n if copies is None else list(copies)
        if len(self.copies) != n:
            _refuse(f"{len(self.copies)} copies for {n} tensors")
        if not all(c is None or isinstance(c, torch.Tensor) for c in self.copies):
            _refuse("a copy is not a tensor")
        types = {c.dtype for c in self.copies if c is not None}
        if len(types) > 1 or types - {torch.bfloat16, torch.float16}:
            _refuse("copies are all bfloat16 or all float16")
        for c, p in zip(self.copies, self.params.tensors):
            if c is not None and (c.numel() != p.numel() or c.device != device or not c.is_contiguous()):
                _refuse("a copy is not contiguous, or has not the size or device of its parameter")

        def each(v, what):
            v = [float(v)] * n if isinstance(v, (int, float)) else [float(x) for x in v]
            if len(v) != n:
                _refuse(f"{len(v)} values of {what} for {n} tensors")
            return v

        def ptr(k, i):
            return self.states[k][i].data_ptr() if k in self.states else None

        second = "v" if state_bits == 32 else "r"
        decay, scale = each(weight_decay, "weight_decay"), each(lr_scale, "lr_scale")
        arr = (ea_adamw_tensor * n)(*[
            ea_adamw_tensor(self.sizes[i], p.data_ptr(), ptr("m", i), ptr(second, i), ptr("m_scale", i), ptr("r_scale", i),
                            None if self.copies[i] is None else self.copies[i].data_ptr(), decay[i], scale[i])
            for i, p in enumerate(self.params.tensors)])
        config = ea_adamw_config(n, _TYPE[self.param_dtype], _TYPE[self.dtype], _TYPE[types.pop()] if types else EA_T_BF16,
                                 state_bits, betas[0], betas[1], eps, seed, step,
                                 ctypes.cast(arr, ctypes.POINTER(ea_adamw_tensor)))
        self._open(config, stream, device)
        self._touched = (*self.params.tensors, *[c for c in self.copies if c is not None],
                         *[t for v in self.states.values() for t in v])
        # one tensor for each count of modifications (pieces of a flat vector have one between them)
        self._modified = tuple({id(b): b for b in (t if t._base is None else t._base for t in self._touched)}.values())

    def step(self, grads, lr: float, clip=None) -> None:
        """One step.  clip: GradNorm's result (the gradients are multiplied by its second value, on the device; a
        step whose factor is NaN is skipped), or None.  A step in a CUDA graph keeps the lr that it was captured with."""
        g = _grad_list(self, grads)
        if clip is not None:
            self._on_device(clip, "clip")
            if clip.dtype != torch.float32 or clip.numel() != 2 or not clip.is_contiguous():
                _refuse("clip is two contiguous float32 values")
        self._call(self._L.ea_adamw_step, (g._ptrs, lr, None if clip is None else clip.data_ptr()),
                   self._touched, g.tensors, () if clip is None else (clip,))
        _C._increment_version(self._modified)

    @property
    def t(self) -> int:
        n = _i64(0)
        with torch.cuda.device(self._index):
            _check(self._L.ea_adamw_step_index(self.h, ctypes.byref(n)))
        return n.value
