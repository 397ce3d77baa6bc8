"""ctypes binding of the language-model operators declared in include/grim_lm.h: layer norm, the gated linear recurrence,
distillation from a teacher's top logits, and the rules for the logits of a served step.

Argument marshalling only, as in binding.py: device buffers are anything with a ``data_ptr()`` or a raw address, dtypes are
"f32" / "f16" / "bf16", leading dimensions count elements, errors are raised as GrimError.  A workspace is a buffer with
``data_ptr()`` and ``nbytes``, or a pair (address, bytes).
"""
from __future__ import annotations

import ctypes
import struct

from .binding import _DT_CODE, GrimError, _addr, _stream, load_library

# struct grim_logit_rules
_RULES = struct.Struct("@PPqiiPPPPPqPq")

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
    "grim_apply_logit_rules": [_P, _I32, _I32, _I64, _I64, _I32, _P, _P, _I64, _P],
}


class _Calls:
    """The library's functions as attributes, bound by the first use of any."""

    def __getattr__(self, name):
        lib = load_library()
        for fn_name, types in ARGTYPES.items():
            fn = getattr(lib, fn_name)
            fn.argtypes = types
            fn.restype = _I64 if fn_name.endswith(("_workspace", "_states")) else _I32
            setattr(self, fn_name, fn)
        return getattr(lib, name)


_c = _Calls()


def _lib():
    return _c


# Marshalling a call for one token costs as much as its kernel takes, so an address is looked up without asking first what kind of
# buffer it is (13 arguments: 6.3 us with _addr and _stream of binding.py, 3.4 with these, on the same CPU).
def _at(buf):
    if buf is None:
        return None
    try:
        return buf.data_ptr()
    except AttributeError:
        return _addr(buf)


def _on(stream):
    try:
        return stream.cuda_stream
    except AttributeError:
        return _stream(stream)


def _room(buf):
    """Address and bytes of a workspace (or None)."""
    if buf is None:
        return None, 0
    if isinstance(buf, tuple):
        return _at(buf[0]), buf[1]
    try:
        return _at(buf), buf.nbytes
    except AttributeError:
        raise TypeError("a workspace has a size: a buffer with nbytes, or (address, bytes)") from None


def layer_norm(x, dtype, ldx: int, gamma, beta, eps: float, N: int, C: int, y, ldy: int, mean=None, rstd=None, stream=None):
    """grim_layer_norm: enqueue y = (x - mean) * rstd * gamma + beta over the rows of x."""
    status = _c.grim_layer_norm(_at(x), _DT_CODE[dtype], ldx, _at(gamma), _at(beta), eps, N, C, _at(y), ldy, _at(mean),
                                _at(rstd), _on(stream))
    if status:
        raise GrimError(status, "grim_layer_norm")


def layer_norm_workspace(N: int, C: int) -> int:
    """grim_layer_norm_workspace: bytes that layer_norm_backward needs."""
    return int(_c.grim_layer_norm_workspace(N, C))


def layer_norm_backward(dy, lddy: int, x, ldx: int, dtype, gamma, mean, rstd, N: int, C: int, dx, lddx: int, dgamma, dbeta,
                        workspace, stream=None):
    """grim_layer_norm_backward: enqueue dx and the column sums dgamma, dbeta (each may be None)."""
    ws, room = _room(workspace)
    status = _c.grim_layer_norm_backward(_at(dy), lddy, _at(x), ldx, _DT_CODE[dtype], _at(gamma), _at(mean), _at(rstd),
                                         N, C, _at(dx), lddx, _at(dgamma), _at(dbeta), ws, room, _on(stream))
    if status:
        raise GrimError(status, "grim_layer_norm_backward")


def glr_states(N: int, H: int) -> int:
    """grim_glr_states: bytes of the states that glr_sequence leaves for its backward pass."""
    return int(_c.grim_glr_states(N, H))


def glr_workspace(N: int, H: int) -> int:
    """grim_glr_workspace: bytes that either direction of glr_sequence needs."""
    return int(_c.grim_glr_workspace(N, H))


def glr_sequence(gates, dtype, ldg: int, bias, h0, seq_start, nseq: int, N: int, H: int, y, ldy: int, h_last, states, workspace,
                 stream=None):
    """grim_glr_sequence: enqueue the gated linear recurrence over N packed rows of gates [forget | candidate | output].
    `states` (a buffer of glr_states bytes, or None) is what the backward pass reads."""
    ws, room = _room(workspace)
    status = _c.grim_glr_sequence(_at(gates), _DT_CODE[dtype], ldg, _at(bias), _at(h0), _at(seq_start), nseq, N, H, _at(y),
                                  ldy, _at(h_last), _at(states), ws, room, _on(stream))
    if status:
        raise GrimError(status, "grim_glr_sequence")


def glr_sequence_backward(gates, dtype, ldg: int, bias, h0, seq_start, nseq: int, N: int, H: int, states, dy, lddy: int, dh_last,
                          dgates, lddg: int, dbias, dh0, workspace, stream=None):
    """grim_glr_sequence_backward: enqueue the gradients of the gates, the bias and the states before the first tokens."""
    ws, room = _room(workspace)
    status = _c.grim_glr_sequence_backward(_at(gates), _DT_CODE[dtype], ldg, _at(bias), _at(h0), _at(seq_start), nseq, N, H,
                                           _at(states), _at(dy), lddy, _at(dh_last), _at(dgates), lddg, _at(dbias),
                                           _at(dh0), ws, room, _on(stream))
    if status:
        raise GrimError(status, "grim_glr_sequence_backward")


def glr_step(gates, ldg: int, bias, h, ldh: int, h_new, ldh_new: int, y, dtype, ldy: int, H: int, batch: int, stream=None):
    """grim_glr_step: one token for `batch` callers; gates 3H x batch and states H x batch in fp32, as grim_lstm_cell has them."""
    status = _c.grim_glr_step(_at(gates), ldg, _at(bias), _at(h), ldh, _at(h_new), ldh_new, _at(y), _DT_CODE[dtype], ldy,
                              H, batch, _on(stream))
    if status:
        raise GrimError(status, "grim_glr_step")


def distill_topk_workspace(N: int, V: int) -> int:
    """grim_distill_topk_workspace: bytes that distill_topk needs."""
    return int(_c.grim_distill_topk_workspace(N, V))


def distill_topk(z, dtype, ldz: int, top_logits, top_ids, k: int, ldt: int, temperature: float, weight, N: int, V: int, loss, dz,
                 lddz: int, workspace, stream=None):
    """grim_distill_topk: enqueue every row's distillation loss and (dz not None) the gradient of their sum."""
    ws, room = _room(workspace)
    status = _c.grim_distill_topk(_at(z), _DT_CODE[dtype], ldz, _at(top_logits), _at(top_ids), k, ldt, temperature,
                                  _at(weight), N, V, _at(loss), _at(dz), lddz, ws, room, _on(stream))
    if status:
        raise GrimError(status, "grim_distill_topk")


def logit_rules(z, dtype, ldz: int, V: int, batch: int, out, ldo: int, *, columns: bool = False, history=None, ld_history: int = 0,
                max_history: int = 0, history_len=None, repetition=None, frequency=None, presence=None, bias_ids=None,
                bias_values=None, nbias: int = 0, ld_bias: int = 0, allowed=None, ld_allowed: int = 0, stream=None):
    """grim_apply_logit_rules: enqueue repetition, frequency and presence penalties, biases and the grammar's mask."""
    rules = _RULES.pack(_at(history) or 0, _at(history_len) or 0, ld_history, max_history, nbias, _at(repetition) or 0,
                        _at(frequency) or 0, _at(presence) or 0, _at(bias_ids) or 0, _at(bias_values) or 0, ld_bias,
                        _at(allowed) or 0, ld_allowed)
    status = _c.grim_apply_logit_rules(_at(z), _DT_CODE[dtype], 1 if columns else 0, ldz, V, batch, rules, _at(out), ldo, _on(stream))
    if status:
        raise GrimError(status, "grim_apply_logit_rules")
