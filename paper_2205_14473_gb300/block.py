"""The operators inside a residual block of a language model (include/ea_block.h): layer norm, a gated linear
recurrence along each sequence and dropout from a counter, each with its gradient.

    norm, scan, drop = LayerNorm(dim, max_rows), GatedScan(dim), Dropout(0.1, seed=7)
    y, stats = norm.forward(x, weight, bias)
    ...                                                  # z and v, products of y
    h, _ = scan.forward(z, v)
    ...                                                  # o, a product of h
    out = drop(o, counter, residual=x)                   # x + dropped-out o

    do = drop.grad(dout, counter)
    dz, dv, _ = scan.grad(dh, z, v, h)
    dx, dw, db = norm.grad(dy, x, stats, weight, add=dout, dw=True, db=True)

Handles, streams, devices and what counts as modified are as in lm.py, and as there nothing has an autograd graph.
Tensors are rows of dim values, with any strides between the rows; a tensor that is read and whose rows are not
contiguous, or that has more than three dimensions and is not contiguous, is copied first.
"""
from __future__ import annotations

import torch

from . import _check
from .block_abi import (ea_dropout_call, ea_dropout_config, ea_layernorm_call, ea_layernorm_config, ea_scan_call,
                        ea_scan_config)
from .lm import _C, _TOKEN, _TYPE, _Handle, _refuse

_F32, _Tensor, _ROWS = torch.float32, torch.Tensor, torch.contiguous_format


def _type(dtype, what) -> int:
    kind = _TYPE.get(dtype)
    if kind is None:
        _refuse(f"{what} is float32, bfloat16 or float16, not {dtype}")
    return kind


class _Block(_Handle):
    """What the three share: checks of rows, and calls that name their tensors only where another stream needs them."""

    def _read(self, t, shape, what):
        """(t or a copy of it, its outer stride, its inner stride) for a tensor of rows that is read."""
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        if t.shape != shape:
            _refuse(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
        stride = t.stride()
        n = len(stride)
        if n == 3 and stride[2] == 1:
            return t, stride[0], stride[1]
        if n > 3:
            return t.contiguous(), 0, shape[-1]
        if n and stride[-1] != 1 and shape[-1] > 1:
            t = t.contiguous()
            stride = t.stride()
        return t, stride[0] if n == 3 else 0, stride[-2] if n > 1 else 0

    def _follows(self, t, shape, what) -> bool:
        """Whether a tensor of rows of this shape is contiguous."""
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        if t.shape != shape:
            _refuse(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
        return t.is_contiguous()

    def _written(self, t, shape, dtype, what):
        """(Its outer stride, its inner stride) for one that is written."""
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        if t.shape != shape:
            _refuse(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
        if t.dtype != dtype:
            _refuse(f"{what} is {t.dtype}, not {dtype}")
        stride = t.stride()
        n = len(stride)
        if n == 3 and stride[2] == 1:
            return stride[0], stride[1]
        if n > 3 and not t.is_contiguous() or n and stride[-1] != 1 and shape[-1] > 1:
            _refuse(f"the rows of {what} are not contiguous")
        return (0, shape[-1]) if n > 3 else (stride[0] if n == 3 else 0, stride[-2] if n > 1 else 0)

    def _values(self, t, shape, dtype, what) -> int:
        """The address of contiguous values of one type."""
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            _refuse(f"{what} is not a contiguous tensor {tuple(shape)} of {dtype}")
        return t.data_ptr()

    def _run(self, f, args, tensors) -> None:
        """As _call; `tensors` may hold None."""
        if (self._only or _C._cuda_getDevice() == self._index) and _C._cuda_getCurrentRawStream(self._index) == self._raw:
            status = f(self.h, *args)
        else:
            status = self._call_from_elsewhere(f, args, [t for t in tensors if t is not None])
        if status:
            _check(status)


def _counts(shape):
    """(outer, inner): rows of a tensor of this shape."""
    n = len(shape)
    if n == 3:
        return shape[0], shape[1]
    if n == 2:
        return 1, shape[0]
    if n == 1:
        return 1, 1
    rows = 1
    for k in shape[:-1]:
        rows *= k
    return 1, rows


class LayerNorm(_Block):
    """Layer norm over rows of dim values, up to max_rows of them a call, and its gradient.

    x, dx and the residual's gradient are of one type; y and dy of the same, or of 16 bits where x is float32; weights
    and their gradients of any of the three types.  Sums and statistics are in 32 bits."""

    _kind = "ea_layernorm"

    def __init__(self, dim: int, max_rows: int, eps: float = 1e-5, stream=None, device=None):
        self.dim, self.max_rows, self.eps = int(dim), int(max_rows), float(eps)
        self._row = torch.Size((self.dim,))
        # The descriptions of a call: of any rows, and of rows one behind another, where only their number changes.
        self._c, d = ea_layernorm_call(), self.dim
        self._flat = ea_layernorm_call(outer=1, x_inner=d, y_inner=d, dx_inner=d, add_inner=d)
        self._open(ea_layernorm_config(self.dim, self.max_rows, self.eps), stream, device)

    def _x(self, x, flat):
        """Describes x's rows; returns the description and what to pass for x.  flat: whether all tensors of the call are
        contiguous."""
        shape = x.shape
        if not shape or shape[-1] != self.dim:
            _refuse(f"x is {tuple(shape)}: its rows are not {self.dim} long")
        if flat:
            c = self._flat
            c.inner = x.numel() // self.dim
        else:
            c = self._c
            c.outer, c.inner = _counts(shape)
            x, c.x_outer, c.x_inner = self._read(x, shape, "x")
        c.x_type = _TYPE.get(x.dtype) or _type(x.dtype, "x")
        return c, x

    def _weight(self, t, c, dtype, what):
        """The address of a weight."""
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        own = t.dtype
        if dtype is not None and own != dtype:
            _refuse(f"{what} is {own}, the other one {dtype}")
        c.weight_type = _TYPE.get(own) or _type(own, what)
        if t.shape != self._row or not t.is_contiguous():
            _refuse(f"{what} is not a contiguous tensor of {self.dim}")
        return t.data_ptr()

    def forward(self, x, weight=None, bias=None, out=None, dtype=None, stats=None):
        """(y, stats): y of x's shape in `dtype` (default: x's) or in `out` (which may be x); stats, of shape
        x.shape[:-1] + (2,), each row's mean and 1 / sqrt(variance + eps), which grad takes, or into `stats`."""
        if not isinstance(x, _Tensor) or x.device != self.device:
            self._on_device(x, "x")
        shape, new = x.shape, out is None
        if not new:
            outer, inner = self._written(out, shape, dtype or getattr(out, "dtype", None), "out")
        flat = x.is_contiguous() and (new or out.is_contiguous())
        c, x = self._x(x, flat)
        w = b = None
        if weight is not None:
            w = self._weight(weight, c, None, "weight")
        if bias is not None:
            b = self._weight(bias, c, None if w is None else weight.dtype, "bias")
        if new:
            kind = dtype or x.dtype
            c.y_type = _TYPE.get(kind) or _type(kind, "out")
            out = torch.empty_like(x, dtype=kind, memory_format=_ROWS)
            outer, inner = c.inner * self.dim, self.dim
        else:
            c.y_type = _type(out.dtype, "out")
        if not flat:
            c.y_outer, c.y_inner = outer, inner
        given = None
        if stats is None:
            stats = x.new_empty((*shape[:-1], 2), dtype=_F32)
            if not new:
                given = (out,)
        else:
            self._values(stats, (*shape[:-1], 2), _F32, "stats")
            given = (stats,) if new else (out, stats)
        self._run(self._L.ea_layernorm_forward, (c, x.data_ptr(), w, b, out.data_ptr(), stats.data_ptr()), (x, weight, bias, out, stats))
        if given:
            _C._increment_version(given)
        return out, stats

    def _sums(self, t, what):
        """A weight's gradient: None (not asked for), True (a new one in 32 bits) or a tensor."""
        if t is None or t is False:
            return None
        if t is True:
            return torch.empty(self._row, dtype=_F32, device=self.device)
        if not isinstance(t, _Tensor) or t.device != self.device:
            self._on_device(t, what)
        if t.shape != self._row or not t.is_contiguous():
            _refuse(f"{what} is not a contiguous tensor of {self.dim}")
        return t

    def grad(self, dy, x, stats, weight=None, add=None, out=None, dw=None, db=None, accumulate: bool = False):
        """(dx, dw, db) from dy = the gradient of forward's y, with its x, stats and weight.  add: rows of x's shape and type
        that are added to dx (the gradient that passes the block by).  dx: into `out` (which may be dy, x or add) or new.
        dw, db: None (not computed), True (new, in 32 bits) or tensors of one type that are written to or, with accumulate, added
        to."""
        if accumulate and (dw is True or db is True):
            _refuse("accumulate needs dw's and db's tensors")
        if not isinstance(x, _Tensor) or x.device != self.device:
            self._on_device(x, "x")
        shape, new, given = x.shape, out is None, []
        if not new:
            outer, inner = self._written(out, shape, x.dtype, "out")
            given.append(out)
        flat = self._follows(dy, shape, "dy") and x.is_contiguous() and (new or out.is_contiguous())
        if add is not None:
            flat = self._follows(add, shape, "add") and flat
            if add.dtype != x.dtype:
                _refuse(f"add is {add.dtype}, x {x.dtype}")
        y = dy
        if not flat:
            y, y_outer, y_inner = self._read(dy, shape, "dy")
            if add is not None:
                add, add_outer, add_inner = self._read(add, shape, "add")
        c, x = self._x(x, flat)
        c.y_type = _TYPE.get(y.dtype) or _type(y.dtype, "dy")
        at = self._values(stats, (*shape[:-1], 2), _F32, "stats")
        w = None if weight is None else self._weight(weight, c, None, "weight")
        if dw is not None:
            if isinstance(dw, _Tensor):
                given.append(dw)
            dw = self._sums(dw, "dw")
        if db is not None:
            if isinstance(db, _Tensor):
                given.append(db)
            db = self._sums(db, "db")
        if dw is not None and db is not None and dw.dtype != db.dtype:
            _refuse(f"dw is {dw.dtype}, db {db.dtype}")
        one = db if dw is None else dw
        if one is not None:
            c.grad_type = _TYPE.get(one.dtype) or _type(one.dtype, "a weight's gradient")
        if new:
            out = torch.empty_like(x, memory_format=_ROWS)
            outer, inner = c.inner * self.dim, self.dim
        if not flat:
            c.y_outer, c.y_inner, c.dx_outer, c.dx_inner = y_outer, y_inner, outer, inner
            if add is not None:
                c.add_outer, c.add_inner = add_outer, add_inner
        self._run(self._L.ea_layernorm_backward,
                  (c, y.data_ptr(), x.data_ptr(), at, w, None if add is None else add.data_ptr(), out.data_ptr(),
                   None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(), int(accumulate)),
                  (y, x, stats, weight, add, out, dw, db))
        if given:
            _C._increment_version(given)
        return out, dw, db


class GatedScan(_Block):
    """The gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) v_t, f = sigmoid(z), in every column of sequences of rows of
    dim values, and its gradient.  z, v, h and their gradients are of one type; states are float32, of shape (batch, dim).  f and 1 - f are
    rounded by themselves: over very many rows of gates that nearly hold, states drift (include/ea_block.h says how far)."""

    _kind = "ea_scan"

    def __init__(self, dim: int, stream=None, device=None):
        self.dim = int(dim)
        self._c = ea_scan_call()
        self._open(ea_scan_config(self.dim), stream, device)

    def _begin(self, z, lengths):
        if not isinstance(z, _Tensor) or z.device != self.device:
            self._on_device(z, "z")
        if z.dim() != 3 or z.shape[2] != self.dim:
            _refuse(f"z is {tuple(z.shape)}, not (batch, length, {self.dim})")
        c = self._c
        c.batch, c.length = z.shape[:2]
        c.type = _type(z.dtype, "z")
        if lengths is None:
            return None
        if not isinstance(lengths, _Tensor) or lengths.device != self.device:
            self._on_device(lengths, "lengths")
        kind = _TOKEN.get(lengths.dtype)
        if kind is None:
            _refuse(f"lengths are int32 or int64, not {lengths.dtype}")
        c.length_type = kind
        if lengths.shape != z.shape[:1]:
            _refuse(f"lengths is {tuple(lengths.shape)}, not ({z.shape[0]},)")
        return lengths.contiguous()

    def _rows(self, t, like, what):
        t, outer, inner = self._read(t, like.shape, what)
        if t.dtype != like.dtype:
            _refuse(f"{what} is {t.dtype}, z {like.dtype}")
        return t, outer, inner

    def _state(self, t, what):
        """(tensor or None, its address or None) of states that are read, or written: None or False, True for a new one."""
        if t is None or t is False:
            return None, None
        shape = (self._c.batch, self.dim)
        if t is True:
            t = torch.empty(shape, dtype=_F32, device=self.device)
            return t, t.data_ptr()
        return t, self._values(t, shape, _F32, what)

    def forward(self, z, v, initial=None, lengths=None, out=None, final=None):
        """(h, final): h of z's shape and type, into `out` (which may be z or v) or new.  initial: the state before the first
        row (None: zeros).  lengths: of the sequences (int32 or int64 on the device; None: all rows): rows behind them get zeros,
        and the state stays as it was.  final: None, True (a new tensor) or a tensor (which may be initial) that receives
        the states after the last rows.  A length outside [0, length] counts as the nearest of the two, and sync() raises for it."""
        given = [t for t in (out, final) if isinstance(t, _Tensor)]
        c, n = self._c, self._begin(z, lengths)
        shape = z.shape
        z, c.z_batch, c.z_row = self._read(z, shape, "z")
        v, c.v_batch, c.v_row = self._rows(v, z, "v")
        initial, first = self._state(initial, "initial")
        final, last = self._state(final, "final")
        if out is None:
            out = torch.empty_like(z, memory_format=_ROWS)
            c.h_batch, c.h_row = shape[1] * self.dim, self.dim
        else:
            c.h_batch, c.h_row = self._written(out, shape, z.dtype, "out")
        self._run(self._L.ea_scan_forward, (c, z.data_ptr(), v.data_ptr(), first, None if n is None else n.data_ptr(), out.data_ptr(), last),
                  (z, v, initial, n, out, final))
        if given:
            _C._increment_version(given)
        return out, final

    def step(self, z, v, state, out=None):
        """One row each of the sequences: z and v of shape (batch, dim).  Updates state (float32) in place and returns h."""
        if not isinstance(z, _Tensor) or z.device != self.device:
            self._on_device(z, "z")
        shape, c, given = z.shape, self._c, out is not None
        if len(shape) != 2 or shape[1] != self.dim:
            _refuse(f"z is {tuple(shape)}, not (batch, {self.dim})")
        kind = z.dtype
        c.type = _TYPE.get(kind) or _type(kind, "z")
        c.batch, c.length = shape[0], 1
        z, _, c.z_batch = self._read(z, shape, "z")
        v, _, c.v_batch = self._rows(v, z, "v")
        at = self._values(state, shape, _F32, "state")
        if not given:
            out = torch.empty_like(z, memory_format=_ROWS)
            c.h_batch = self.dim
        else:
            _, c.h_batch = self._written(out, shape, kind, "out")
        c.z_row = c.v_row = c.h_row = self.dim
        self._run(self._L.ea_scan_forward, (c, z.data_ptr(), v.data_ptr(), at, None, out.data_ptr(), at), (z, v, state, out))
        _C._increment_version((out, state) if given else (state,))
        return out

    def grad(self, dh, z, v, h, initial=None, lengths=None, d_final=None, dz=None, dv=None, d_initial=None):
        """(dz, dv, d_initial) from dh = the gradient of forward's h and d_final = that of its final states (None: zeros), with
        its z, v, h, initial and lengths.  dz (which may be z or dh) and dv (v or dh) are written to, or new.  d_initial: None,
        True (a new tensor) or a tensor (which may be d_final)."""
        given = [t for t in (dz, dv, d_initial) if isinstance(t, _Tensor)]
        c, n = self._c, self._begin(z, lengths)
        shape = z.shape
        z, c.z_batch, c.z_row = self._read(z, shape, "z")
        dh, c.dh_batch, c.dh_row = self._rows(dh, z, "dh")
        v, c.v_batch, c.v_row = self._rows(v, z, "v")
        h, c.h_batch, c.h_row = self._rows(h, z, "h")
        initial, first = self._state(initial, "initial")
        d_final, last = self._state(d_final, "d_final")
        d_initial, d_first = self._state(d_initial, "d_initial")
        if dz is None:
            dz = torch.empty_like(z, memory_format=_ROWS)
            c.dz_batch, c.dz_row = shape[1] * self.dim, self.dim
        else:
            c.dz_batch, c.dz_row = self._written(dz, shape, z.dtype, "dz")
        if dv is None:
            dv = torch.empty_like(z, memory_format=_ROWS)
            c.dv_batch, c.dv_row = shape[1] * self.dim, self.dim
        else:
            c.dv_batch, c.dv_row = self._written(dv, shape, z.dtype, "dv")
        self._run(self._L.ea_scan_backward,
                  (c, dh.data_ptr(), z.data_ptr(), v.data_ptr(), h.data_ptr(), first, None if n is None else n.data_ptr(), last,
                   dz.data_ptr(), dv.data_ptr(), d_first),
                  (dh, z, v, h, initial, n, d_final, dz, dv, d_initial))
        if given:
            _C._increment_version(given)
        return dz, dv, d_initial

    def sync(self) -> None:
        with torch.cuda.device(self._index):
            _check(self._L.ea_scan_sync_status(self.h))


class Dropout(_Block):
    """Dropout whose mask is a function of (seed, counter, element) and is stored nowhere: the gradient draws it again.

    p: the probability that an element is dropped, as the nearest multiple of 2^-16 (self.p).  The mask of a call goes by
    `counter`, an integer in [0, 2^64) or an int64 tensor of one value on the device, which a captured graph reads at every
    replay: another one for every call of a training step (step * layers + layer, say).  Use another seed than an optimizer's."""

    _kind = "ea_dropout"

    def __init__(self, p: float, seed: int = 0, stream=None, device=None):
        self.seed = int(seed)
        if not 0 <= self.seed < 1 << 64:
            _refuse("seed is outside [0, 2^64)")
        self._c, self._flat = ea_dropout_call(), ea_dropout_call(outer=1, inner=1)
        self._open(ea_dropout_config(float(p), self.seed), stream, device)
        self.p = round(65536 * float(p)) / 65536

    def __call__(self, x, counter, residual=None, out=None, dtype=None):
        """residual + x / (1 - p) where an element is kept, residual (or 0) where it is not, of x's shape, in `dtype` (default:
        the residual's type, or x's) or into `out` (which may be x or residual).  x and the result are of one type, or one of them
        float32; residual is of the result's."""
        given = out is not None
        if not isinstance(x, _Tensor) or x.device != self.device:
            self._on_device(x, "x")
        shape = x.shape
        if not shape:
            _refuse("x has no dimensions")
        if dtype is None:
            dtype = (out if given else residual if residual is not None else x).dtype
        if given:
            outer, inner = self._written(out, shape, dtype, "out")
        flat = x.is_contiguous() and (not given or out.is_contiguous())
        if residual is not None:
            flat = self._follows(residual, shape, "residual") and flat
            if residual.dtype != dtype:
                _refuse(f"residual is {residual.dtype}, the result {dtype}")
        if flat:
            c = self._flat
            c.dim = x.numel()
        else:
            c = self._c
            c.outer, c.inner = _counts(shape)
            c.dim = shape[-1]
            x, c.x_outer, c.x_inner = self._read(x, shape, "x")
            if residual is not None:
                residual, c.add_outer, c.add_inner = self._read(residual, shape, "residual")
            c.y_outer, c.y_inner = (outer, inner) if given else (c.inner * c.dim, c.dim)
        c.x_type, c.y_type = _TYPE.get(x.dtype) or _type(x.dtype, "x"), _TYPE.get(dtype) or _type(dtype, "the result")
        if not given:
            out = torch.empty_like(x, dtype=dtype, memory_format=_ROWS)
        if isinstance(counter, _Tensor):
            if counter.device != self.device or counter.dtype != torch.int64 or counter.numel() != 1:
                _refuse(f"counter is an integer or an int64 tensor of one value on {self.device}")
            number, at = 0, counter.data_ptr()
        else:
            number, at = int(counter), None
            if not 0 <= number < 1 << 64:
                _refuse("counter is outside [0, 2^64)")
        self._run(self._L.ea_dropout_apply, (c, x.data_ptr(), None if residual is None else residual.data_ptr(), number, at, out.data_ptr()),
                  (x, residual, out, counter if at is not None else None))
        if given:
            _C._increment_version((out,))
        return out

    def grad(self, dy, counter, out=None, dtype=None):
        """The gradient of x from dy = that of the result of the call with this counter, in `dtype` (x's; default: dy's) or into
        `out`.  The residual's gradient is dy."""
        return self(dy, counter, out=out, dtype=dtype)
