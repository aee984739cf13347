"""The C structures and functions of include/ea_block.h, same names (ctypes)."""
from __future__ import annotations

import ctypes

from .lm_abi import _f32, _i32, _i64, _P

_u64 = ctypes.c_uint64


class ea_layernorm_config(ctypes.Structure):
    _fields_ = [("dim", _i64), ("max_rows", _i64), ("eps", _f32)]


class ea_layernorm_call(ctypes.Structure):
    _fields_ = [("outer", _i64), ("inner", _i64), ("x_outer", _i64), ("x_inner", _i64), ("y_outer", _i64), ("y_inner", _i64),
                ("dx_outer", _i64), ("dx_inner", _i64), ("add_outer", _i64), ("add_inner", _i64), ("x_type", _i32), ("y_type", _i32),
                ("weight_type", _i32), ("grad_type", _i32)]


class ea_scan_config(ctypes.Structure):
    _fields_ = [("dim", _i64)]


class ea_scan_call(ctypes.Structure):
    _fields_ = [("batch", _i64), ("length", _i64), ("z_batch", _i64), ("z_row", _i64), ("v_batch", _i64), ("v_row", _i64),
                ("h_batch", _i64), ("h_row", _i64), ("dh_batch", _i64), ("dh_row", _i64), ("dz_batch", _i64), ("dz_row", _i64),
                ("dv_batch", _i64), ("dv_row", _i64), ("type", _i32), ("length_type", _i32)]


class ea_dropout_config(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", _u64)]


class ea_dropout_call(ctypes.Structure):
    _fields_ = [("outer", _i64), ("inner", _i64), ("dim", _i64), ("x_outer", _i64), ("x_inner", _i64), ("add_outer", _i64),
                ("add_inner", _i64), ("y_outer", _i64), ("y_inner", _i64), ("x_type", _i32), ("y_type", _i32)]


def declare(L) -> None:
    """The argument types of include/ea_block.h's functions."""
    size, handle = ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(_P)
    for name, config in (("ea_layernorm", ea_layernorm_config), ("ea_scan", ea_scan_config), ("ea_dropout", ea_dropout_config)):
        getattr(L, name + "_workspace_bytes").argtypes = [ctypes.POINTER(config), size]
        getattr(L, name + "_init").argtypes = [ctypes.POINTER(config), _P, ctypes.c_size_t, _P, handle]
        getattr(L, name + "_destroy").argtypes = [_P]
    L.ea_layernorm_forward.argtypes = [_P, ctypes.POINTER(ea_layernorm_call), _P, _P, _P, _P, _P]
    L.ea_layernorm_backward.argtypes = [_P, ctypes.POINTER(ea_layernorm_call), _P, _P, _P, _P, _P, _P, _P, _P, _i32]
    L.ea_scan_forward.argtypes = [_P, ctypes.POINTER(ea_scan_call), _P, _P, _P, _P, _P, _P]
    L.ea_scan_backward.argtypes = [_P, ctypes.POINTER(ea_scan_call), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.ea_scan_sync_status.argtypes = [_P]
    L.ea_scan_selftest_exchange.argtypes = [_i64, _i32, _P, ctypes.POINTER(_i32)]
    L.ea_dropout_apply.argtypes = [_P, ctypes.POINTER(ea_dropout_call), _P, _P, _u64, _P, _P]


EXPORTED = [f"{n}_{f}" for n in ("ea_layernorm", "ea_scan", "ea_dropout") for f in ("workspace_bytes", "init", "destroy")] + [
    "ea_layernorm_forward", "ea_layernorm_backward", "ea_scan_forward", "ea_scan_backward", "ea_scan_sync_status", "ea_scan_selftest_exchange",
    "ea_dropout_apply"]
