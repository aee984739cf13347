"""The C structures and functions of include/ea_lm.h, same names (ctypes)."""
from __future__ import annotations

import ctypes

EA_T_F32, EA_T_BF16, EA_T_F16, EA_T_I32, EA_T_I64 = range(5)
EA_ADAMW_BLOCK = 256
_P, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class ea_embed_config(ctypes.Structure):
    _fields_ = [("vocab", _i64), ("dim", _i64), ("max_tokens", _i64), ("padding", _i64), ("scale", _f32)]


class ea_embed_call(ctypes.Structure):
    _fields_ = [("outer", _i64), ("inner", _i64), ("token_outer", _i64), ("token_inner", _i64), ("row_outer", _i64),
                ("row_inner", _i64), ("table_stride", _i64), ("token_type", _i32), ("row_type", _i32),
                ("table_type", _i32)]


class ea_grad_norm_config(ctypes.Structure):
    _fields_ = [("n_tensors", _i32), ("grad_type", _i32), ("sizes", ctypes.POINTER(_i64))]


class ea_adamw_tensor(ctypes.Structure):
    _fields_ = [("size", _i64), ("param", _P), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P), ("copy", _P),
                ("weight_decay", _f32), ("lr_scale", _f32)]


class ea_adamw_config(ctypes.Structure):
    _fields_ = [("n_tensors", _i32), ("param_type", _i32), ("grad_type", _i32), ("copy_type", _i32),
                ("state_bits", _i32), ("beta1", _f32), ("beta2", _f32), ("eps", _f32), ("seed", ctypes.c_uint64),
                ("step", _i64), ("tensors", ctypes.POINTER(ea_adamw_tensor))]


def declare(L) -> None:
    """The argument types of include/ea_lm.h's functions."""
    size, handle = ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(_P)
    for name, config in (("ea_embed", ea_embed_config), ("ea_grad_norm", ea_grad_norm_config),
                         ("ea_adamw", ea_adamw_config)):
        getattr(L, name + "_workspace_bytes").argtypes = [ctypes.POINTER(config), size]
        getattr(L, name + "_init").argtypes = [ctypes.POINTER(config), _P, ctypes.c_size_t, _P, handle]
        getattr(L, name + "_destroy").argtypes = [_P]
    L.ea_embed_lookup.argtypes = [_P, ctypes.POINTER(ea_embed_call), _P, _P, _P]
    L.ea_embed_grad.argtypes = [_P, ctypes.POINTER(ea_embed_call), _P, _P, _P, _i32]
    L.ea_embed_sync_status.argtypes = [_P]
    L.ea_grad_norm.argtypes = [_P, _P, _f32, _f32, _P]
    L.ea_adamw_step.argtypes = [_P, _P, _f32, _P]
    L.ea_adamw_step_index.argtypes = [_P, ctypes.POINTER(_i64)]
    L.ea_adamw_selftest_sqrt.argtypes = [_P, ctypes.POINTER(ctypes.c_uint64)]


EXPORTED = [f"{n}_{f}" for n in ("ea_embed", "ea_grad_norm", "ea_adamw") for f in ("workspace_bytes", "init", "destroy")] + [
    "ea_embed_lookup", "ea_embed_grad", "ea_embed_sync_status", "ea_grad_norm", "ea_adamw_step", "ea_adamw_step_index",
    "ea_adamw_selftest_sqrt"]
