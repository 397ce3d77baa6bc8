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
    "grim_glr_states": [_I64, _I64],
    "grim_glr_workspace": [_I64, _I64],
    "grim_glr_sequence": [_P, _I32, _I64, _P, _P, _P, _I32, _I64, _I64, _P, _I64, _P, _P, _P, _I64, _P],
    "grim_glr_sequence_backward": [_P, _I32, _I64, _P, _P, _P, _I32, _I64, _I64, _P, _P, _I64, _P, _P, _I64, _P, _P, _P, _I64, _P],
    "grim_glr_step": [_P, _I64, _P, _P, _I64, _P, _I64, _P, _I32, _I64, _I64, _I32, _P],
    "grim_distill_topk_workspace": [_I64, _I64],
    "grim_distill_topk": [_P, _I32, _I64, _P, _P, _I32, _I64, _F, _P, _I64, _I64, _P, _P, _I64, _P, _I64, _P],
    "grim_apply_logit_rules": [_P, _I32, _I32, _I64, _I64, _I32, ctypes.POINTER(LogitRules), _P, _I64, _P],
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


def glr_states(N: int, H: int) -> int:
    """grim_glr_states: bytes of the states that glr_sequence leaves for its backward pass."""
    return int(_lib().grim_glr_states(N, H))


def glr_workspace(N: int, H: int) -> int:
    """grim_glr_workspace: bytes that either direction of glr_sequence needs."""
    return int(_lib().grim_glr_workspace(N, H))


def glr_sequence(gates, dtype, ldg: int, bias, h0, seq_start, nseq: int, N: int, H: int, y, ldy: int, h_last, states, workspace,
                 stream=None):
    """grim_glr_sequence: enqueue the gated linear recurrence over N packed rows of gates [forget | candidate | output].
    `states` (a buffer of glr_states bytes, or None) is what the backward pass reads."""
    ws, room = _room(workspace)
    _check(_lib().grim_glr_sequence(_addr(gates), _DT_CODE[dtype], ldg, _addr(bias), _addr(h0), _addr(seq_start), nseq, N, H, _addr(y),
                                    ldy, _addr(h_last), _addr(states), ws, room, _stream(stream)), "grim_glr_sequence")


def glr_sequence_backward(gates, dtype, ldg: int, bias, h0, seq_start, nseq: int, N: int, H: int, states, dy, lddy: int, dh_last,
                          dgates, lddg: int, dbias, dh0, workspace, stream=None):
    """grim_glr_sequence_backward: enqueue the gradients of the gates, the bias and the states before the first tokens."""
    ws, room = _room(workspace)
    _check(_lib().grim_glr_sequence_backward(_addr(gates), _DT_CODE[dtype], ldg, _addr(bias), _addr(h0), _addr(seq_start), nseq, N, H,
                                             _addr(states), _addr(dy), lddy, _addr(dh_last), _addr(dgates), lddg, _addr(dbias),
                                             _addr(dh0), ws, room, _stream(stream)), "grim_glr_sequence_backward")


def glr_step(gates, ldg: int, bias, h, ldh: int, h_new, ldh_new: int, y, dtype, ldy: int, H: int, batch: int, stream=None):
    """grim_glr_step: one token for `batch` callers; gates 3H x batch and states H x batch in fp32, as grim_lstm_cell has them."""
    _check(_lib().grim_glr_step(_addr(gates), ldg, _addr(bias), _addr(h), ldh, _addr(h_new), ldh_new, _addr(y), _DT_CODE[dtype], ldy,
                                H, batch, _stream(stream)), "grim_glr_step")


def distill_topk_workspace(N: int, V: int) -> int:
    """grim_distill_topk_workspace: bytes that distill_topk needs."""
    return int(_lib().grim_distill_topk_workspace(N, V))


def distill_topk(z, dtype, ldz: int, top_logits, top_ids, k: int, ldt: int, temperature: float, weight, N: int, V: int, loss, dz,
                 lddz: int, workspace, stream=None):
    """grim_distill_topk: enqueue every row's distillation loss and (dz not None) the gradient of their sum."""
    ws, room = _room(workspace)
    _check(_lib().grim_distill_topk(_addr(z), _DT_CODE[dtype], ldz, _addr(top_logits), _addr(top_ids), k, ldt, temperature,
                                    _addr(weight), N, V, _addr(loss), _addr(dz), lddz, ws, room, _stream(stream)),
           "grim_distill_topk")


def logit_rules(z, dtype, ldz: int, V: int, batch: int, out, ldo: int, *, columns: bool = False, history=None, ld_history: int = 0,
                max_history: int = 0, history_len=None, repetition=None, frequency=None, presence=None, bias_ids=None,
                bias_values=None, nbias: int = 0, ld_bias: int = 0, allowed=None, ld_allowed: int = 0, stream=None):
    """grim_apply_logit_rules: enqueue repetition, frequency and presence penalties, biases and the grammar's mask."""
    rules = LogitRules(_addr(history), _addr(history_len), ld_history, max_history, nbias, _addr(repetition), _addr(frequency),
                       _addr(presence), _addr(bias_ids), _addr(bias_values), ld_bias, _addr(allowed), ld_allowed)
    _check(_lib().grim_apply_logit_rules(_addr(z), _DT_CODE[dtype], int(bool(columns)), ldz, V, batch, ctypes.byref(rules), _addr(out),
                                         ldo, _stream(stream)), "grim_apply_logit_rules")
