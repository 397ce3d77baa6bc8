"""ctypes binding of the language-model operators declared in include/grim_lm.h: layer norm, the gated linear recurrence,
distillation from a teacher's top logits, and the rules for the logits of a served step.

Argument marshalling only, as in binding.py: device buffers are anything with a ``data_ptr()`` or a raw address, dtypes are
"f32" / "f16" / "bf16", leading dimensions count elements, errors are raised as GrimError.
"""
from __future__ import annotations

import ctypes

from .binding import _DT_CODE, _addr, _check, _stream, load_library

_bound = None


class LogitRules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_len", ctypes.c_void_p), ("ld_history", ctypes.c_int64),
                ("max_history", ctypes.c_int32), ("nbias", ctypes.c_int32),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p), ("ld_bias", ctypes.c_int64),
                ("allowed", ctypes.c_void_p), ("ld_allowed", ctypes.c_int64)]


_I64, _I32, _P, _F = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float
ARGTYPES = {
    "grim_layer_norm": [_P, _I32, _I64, _P, _P, _F, _I64, _I64, _P, _I64, _P, _P, _P],
    "grim_layer_norm_backward": [_P, _I64, _P, _I64, _I32, _P, _P, _P, _I64, _I64, _P, _I64, _P, _P, _P, _I64, _P],
    "grim_layer_norm_workspace": [_I64, _I64],
}


def _lib():
    global _bound
    if _bound is None:
        lib = load_library()
        for name, types in ARGTYPES.items():
            fn = getattr(lib, name)
            fn.argtypes = types
            fn.restype = _I64 if name.endswith(("_workspace", "_states")) else _I32
        _bound = lib
    return _bound


def _room(buf):
    """Address and bytes of a workspace tensor (or None)."""
    return (None, 0) if buf is None else (_addr(buf), buf.numel() * buf.element_size())


def layer_norm(x, dtype, ldx: int, gamma, beta, eps: float, N: int, C: int, y, ldy: int, mean=None, rstd=None, stream=None):
    """grim_layer_norm: enqueue y = (x - mean) * rstd * gamma + beta over the rows of x."""
    _check(_lib().grim_layer_norm(_addr(x), _DT_CODE[dtype], ldx, _addr(gamma), _addr(beta), eps, N, C, _addr(y), ldy, _addr(mean),
                                  _addr(rstd), _stream(stream)), "grim_layer_norm")


def layer_norm_workspace(N: int, C: int) -> int:
    """grim_layer_norm_workspace: bytes that layer_norm_backward needs."""
    return int(_lib().grim_layer_norm_workspace(N, C))


def layer_norm_backward(dy, lddy: int, x, ldx: int, dtype, gamma, mean, rstd, N: int, C: int, dx, lddx: int, dgamma, dbeta,
                        workspace, stream=None):
    """grim_layer_norm_backward: enqueue dx and the column sums dgamma, dbeta (each may be None)."""
    ws, room = _room(workspace)
    _check(_lib().grim_layer_norm_backward(_addr(dy), lddy, _addr(x), ldx, _DT_CODE[dtype], _addr(gamma), _addr(mean), _addr(rstd),
                                           N, C, _addr(dx), lddx, _addr(dgamma), _addr(dbeta), ws, room, _stream(stream)),
           "grim_layer_norm_backward")
