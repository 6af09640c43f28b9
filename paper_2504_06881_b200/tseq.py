"""Thin ctypes binding over the sequence and storage entry points of libtconv.so (include/tconv.h): 8-bit activations,
gated linear recurrence, root-mean-square norm.

Argument marshalling only; every step runs in the library's CUDA kernels.  Tensors go as they are (device pointers) and
the functions return the status; ``nn`` has the checked forms with autograd.
"""
from __future__ import annotations

import ctypes

from .tconv import DTYPES, _lib, _p, _stream


class ScanDesc(ctypes.Structure):
    """tconv_scan_desc_t."""
    _fields_ = [("N", ctypes.c_int32), ("C", ctypes.c_int32), ("L", ctypes.c_int64), ("dtype", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("x_batch", "x_row", "gate_batch", "gate_row", "grad_batch")]


class NormDesc(ctypes.Structure):
    """tconv_norm_desc_t."""
    _fields_ = [("N", ctypes.c_int32), ("C", ctypes.c_int32), ("P", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


def _bind():
    vp, sz, i64, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int
    sd, nd = ctypes.POINTER(ScanDesc), ctypes.POINTER(NormDesc)
    for name, res, args in (
            ("tconv_q8_codes_bytes", sz, [i64, i64]), ("tconv_q8_scales_bytes", sz, [i64, i64]),
            ("tconv_q8_store", ci, [i64, i64, ci] + [vp] * 4), ("tconv_q8_restore", ci, [i64, i64, ci] + [vp] * 4),
            ("tconv_scan_states_bytes", sz, [sd]), ("tconv_scan_workspace_bytes", sz, [sd, ci]),
            ("tconv_scan_forward", ci, [sd] + [vp] * 12 + [sz, vp]),
            ("tconv_scan_backward", ci, [sd] + [vp] * 14 + [sz, vp]),
            ("tconv_norm_workspace_bytes", sz, [nd]),
            ("tconv_norm_forward", ci, [nd] + [vp] * 11), ("tconv_norm_backward", ci, [nd] + [vp] * 10 + [sz, vp])):
        fn = getattr(_lib, name)
        fn.restype, fn.argtypes = res, args


_bind()


def scan_desc(N, C, L, dtype="f32", x_batch=None, x_row=None, gate_batch=None, gate_row=None, grad_batch=None) -> ScanDesc:
    """Strides left out are those of dense tensors [N, C, L]."""
    v = lambda given, dense: dense if given is None else given
    return ScanDesc(N, C, L, DTYPES[dtype], v(x_batch, C * L), v(x_row, L), v(gate_batch, C * L), v(gate_row, L),
                    v(grad_batch, C * L))


def norm_desc(N, C, P, dtype="f32", eps=1e-6) -> NormDesc:
    return NormDesc(N, C, P, DTYPES[dtype], eps)


def _bytes(t):
    return 0 if t is None else t.numel() * t.element_size()


# ---- the C entry points, one to one ------------------------------------------------
def tconv_q8_codes_bytes(rows: int, inner: int) -> int:
    return int(_lib.tconv_q8_codes_bytes(rows, inner))


def tconv_q8_scales_bytes(rows: int, inner: int) -> int:
    return int(_lib.tconv_q8_scales_bytes(rows, inner))


def tconv_q8_store(rows, inner, dtype, x, codes, scales, stream=None) -> int:
    return _lib.tconv_q8_store(rows, inner, DTYPES[dtype], _p(x), _p(codes), _p(scales), _stream(stream))


def tconv_q8_restore(rows, inner, dtype, codes, scales, x, stream=None) -> int:
    return _lib.tconv_q8_restore(rows, inner, DTYPES[dtype], _p(codes), _p(scales), _p(x), _stream(stream))


def tconv_scan_states_bytes(d: ScanDesc) -> int:
    return int(_lib.tconv_scan_states_bytes(ctypes.byref(d)))


def tconv_scan_workspace_bytes(d: ScanDesc, backward: bool) -> int:
    return int(_lib.tconv_scan_workspace_bytes(ctypes.byref(d), int(backward)))


def tconv_scan_forward(d: ScanDesc, x, gate, h0, lengths, y, h_last, states=None, kept=(None,) * 4, workspace=None,
                       stream=None) -> int:
    """kept: codes and scales of x, then of gate."""
    return _lib.tconv_scan_forward(ctypes.byref(d), *map(_p, (x, gate, h0, lengths, y, h_last, states, *kept, workspace)),
                                   _bytes(workspace), _stream(stream))


def tconv_scan_backward(d: ScanDesc, x, gate, lengths, states, grad_y, grad_h_last, grad_x, grad_gate, grad_h0=None,
                        kept=(None,) * 4, workspace=None, stream=None) -> int:
    return _lib.tconv_scan_backward(ctypes.byref(d), *map(_p, (x, gate, *kept, lengths, states, grad_y, grad_h_last, grad_x,
                                                               grad_gate, grad_h0, workspace)),
                                    _bytes(workspace), _stream(stream))


def tconv_norm_workspace_bytes(d: NormDesc) -> int:
    return int(_lib.tconv_norm_workspace_bytes(ctypes.byref(d)))


def tconv_norm_forward(d: NormDesc, x, residual, weight, sum, y, rstd=None, y_q8=(None, None), s_q8=(None, None),
                       stream=None) -> int:
    return _lib.tconv_norm_forward(ctypes.byref(d), *map(_p, (x, residual, weight, sum, y, rstd, *y_q8, *s_q8)),
                                   _stream(stream))


def tconv_norm_backward(d: NormDesc, s, rstd, weight, grad_y, grad_sum, grad_x, grad_weight=None, s_q8=(None, None),
                        workspace=None, stream=None) -> int:
    return _lib.tconv_norm_backward(ctypes.byref(d), *map(_p, (s, *s_q8, rstd, weight, grad_y, grad_sum, grad_x, grad_weight,
                                                               workspace)), _bytes(workspace), _stream(stream))
