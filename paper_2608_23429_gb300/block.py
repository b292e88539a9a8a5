"""ctypes binding of the full step's operators (``include/chebboost_block.h``), same names, marshalling only.

The operators live in libchebboost with the rest; pointers, streams, errors and
constants are those of :mod:`paper_2608_23429_gb300.chebboost`.
"""
from __future__ import annotations

import ctypes

from .chebboost import CB_BF16, CbError, _lib, _stream

_P, _I, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64


def _addr(x):
    """Address of a buffer (tensor, int or None). These calls take a few microseconds in all, so this is kept short."""
    return x if x is None or x.__class__ is int else x.data_ptr()


def _raise(rc: int, call: str):
    raise CbError(rc, call)


class cb_norm_desc(ctypes.Structure):
    """Sizes and types of :func:`cb_norm_residual`; strides of 0 mean contiguous."""
    _fields_ = [("rows", _L), ("hidden", _L), ("tokens", _L), ("x_stride", _L), ("branch_stride", _L),
                ("x_out_stride", _L), ("out_stride", _L), ("line_stride", _L), ("x_dtype", _I), ("branch_dtype", _I),
                ("param_dtype", _I), ("out_dtype", _I), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


class cb_linear_desc(ctypes.Structure):
    """A layer, as :func:`cb_linear_create` fills it in."""
    _fields_ = [("in_features", _L), ("out_features", _L), ("w_stride", _L), ("type", _I), ("bias_dtype", _I),
                ("activation", ctypes.c_int32), ("reserved", ctypes.c_int32), ("w", _P), ("w_scale", _P), ("bias", _P)]


class cb_linear_io(ctypes.Structure):
    """Sizes and types of one :func:`cb_linear_run`; strides of 0 mean contiguous."""
    _fields_ = [("rows", _L), ("tokens", _L), ("x_stride", _L), ("out_stride", _L), ("resid_stride", _L),
                ("resid_out_stride", _L), ("gate_stride", _L), ("out_dtype", _I), ("resid_dtype", _I), ("gate_dtype", _I),
                ("reserved", ctypes.c_int32)]


CB_ACT_NONE, CB_ACT_GELU, CB_ACT_SILU = 0, 1, 2
CB_MAX_IN_FEATURES = 1 << 22

_sig = {
    "cb_norm_residual": ([_P] * 11, _I),
    "cb_linear_create": ([_P, ctypes.POINTER(_P)], _I),
    "cb_linear_destroy": ([_P], None),
    "cb_linear_set_option": ([_P, _I, _L], _I),
    "cb_linear_run": ([_P] * 9, _I),
    "cb_linear_device_status": ([_P, _P], _I),
}
for _name, (_args, _res) in _sig.items():
    _f = getattr(_lib, _name)
    _f.argtypes, _f.restype = _args, _res

EXPORTED = tuple(_sig)
_norm_residual, _linear_run = _lib.cb_norm_residual, _lib.cb_linear_run


def cb_norm_residual(desc: cb_norm_desc, x, branch=None, gate=None, weight=None, scale=None, shift=None, x_out=None,
                     out=None, out_scale=None, stream=None) -> None:
    """RMS norm of ``x + gate * branch`` into ``out`` (with ``out_scale`` where it is e4m3), the sum into ``x_out``."""
    rc = _norm_residual(ctypes.addressof(desc), _addr(x), _addr(branch), _addr(gate), _addr(weight), _addr(scale), _addr(shift),
                        _addr(x_out), _addr(out), _addr(out_scale), None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_norm_residual")


def cb_linear_create(w, out_features: int, in_features: int, type: int, w_scale=None, bias=None,
                     bias_dtype: int = CB_BF16, activation: int = CB_ACT_NONE, w_stride: int = 0):
    """The layer's handle. The library keeps addresses only: the caller keeps the buffers."""
    d = cb_linear_desc(in_features, out_features, w_stride, type, bias_dtype, activation, 0, _addr(w), _addr(w_scale),
                       _addr(bias))
    layer = _P()
    rc = _lib.cb_linear_create(ctypes.addressof(d), ctypes.byref(layer))
    if rc < 0:
        _raise(rc, "cb_linear_create")
    return layer


def cb_linear_destroy(layer) -> None:
    _lib.cb_linear_destroy(layer)


def cb_linear_set_option(layer, option: int, value: int) -> None:
    rc = _lib.cb_linear_set_option(layer, option, int(value))
    if rc < 0:
        _raise(rc, "cb_linear_set_option")


def cb_linear_run(layer, io: cb_linear_io, x, x_scale=None, resid=None, gate=None, out=None, resid_out=None,
                  stream=None) -> None:
    """``act(x w^T + bias)`` into ``out`` and/or, gated and added to ``resid``, into ``resid_out``."""
    rc = _linear_run(layer, ctypes.addressof(io), _addr(x), _addr(x_scale), _addr(resid), _addr(gate), _addr(out),
                     _addr(resid_out), None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_linear_run")


def cb_linear_device_status(stream=None) -> int:
    st = ctypes.c_int(0)
    rc = _lib.cb_linear_device_status(ctypes.addressof(st), _stream(stream))
    if rc < 0:
        _raise(rc, "cb_linear_device_status")
    return st.value
