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


class cb_norm_around_desc(ctypes.Structure):
    """Sizes and types of :func:`cb_norm_around`; strides of 0 mean contiguous. Made by name, its factors are 1."""
    _fields_ = [("rows", _L), ("hidden", _L), ("tokens", _L), ("x_stride", _L), ("branch_stride", _L),
                ("x_out_stride", _L), ("out_stride", _L), ("line_stride", _L), ("x_dtype", _I), ("branch_dtype", _I),
                ("param_dtype", _I), ("out_dtype", _I), ("after", ctypes.c_int32), ("before", ctypes.c_int32),
                ("after_eps", ctypes.c_float), ("before_eps", ctypes.c_float), ("x_factor", ctypes.c_float),
                ("branch_factor", ctypes.c_float), ("reserved", ctypes.c_int32)]

    def __init__(self, *args, **kw):
        if not args:
            kw = {"x_factor": 1.0, "branch_factor": 1.0, **kw}
        super().__init__(*args, **kw)


class cb_mx_desc(ctypes.Structure):
    """Sizes and types of :func:`cb_mx_quantize` and :func:`cb_mx_dequantize`; strides of 0 mean contiguous."""
    _fields_ = [("rows", _L), ("features", _L), ("stride", _L), ("codes_stride", _L), ("dtype", _I),
                ("reserved", ctypes.c_int32)]


class cb_linear_desc(ctypes.Structure):
    """A layer, as :func:`cb_linear_create` fills it in."""
    _fields_ = [("in_features", _L), ("out_features", _L), ("w_stride", _L), ("type", _I), ("bias_dtype", _I),
                ("activation", ctypes.c_int32), ("reserved", ctypes.c_int32), ("w", _P), ("w_scale", _P), ("bias", _P)]


class cb_linear_io(ctypes.Structure):
    """Sizes and types of one :func:`cb_linear_run`; strides of 0 mean contiguous. ``out_scale`` is an address."""
    _fields_ = [("rows", _L), ("tokens", _L), ("x_stride", _L), ("out_stride", _L), ("resid_stride", _L),
                ("resid_out_stride", _L), ("gate_stride", _L), ("out_dtype", _I), ("resid_dtype", _I), ("gate_dtype", _I),
                ("reserved", ctypes.c_int32), ("out_scale", _P)]


CB_ACT_NONE, CB_ACT_GELU, CB_ACT_SILU = 0, 1, 2
CB_NORM_NONE, CB_NORM_RMS, CB_NORM_LAYER = 0, 1, 2
CB_MAX_IN_FEATURES = 1 << 22
CB_MX_BLOCK = 32

_sig = {
    "cb_norm_residual": ([_P] * 11, _I),
    "cb_norm_around": ([_P] * 14, _I),
    "cb_mx_scale_bytes": ([_L, _L, _P], _I),
    "cb_mx_quantize": ([_P] * 5, _I),
    "cb_mx_dequantize": ([_P] * 5, _I),
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
_norm_around = _lib.cb_norm_around
_mx_quantize, _mx_dequantize = _lib.cb_mx_quantize, _lib.cb_mx_dequantize


def cb_norm_residual(desc: cb_norm_desc, x, branch=None, gate=None, weight=None, scale=None, shift=None, x_out=None,
                     out=None, out_scale=None, stream=None) -> None:
    """RMS norm of ``x + gate * branch`` into ``out`` (with ``out_scale`` where it is e4m3), the sum into ``x_out``."""
    rc = _norm_residual(ctypes.addressof(desc), _addr(x), _addr(branch), _addr(gate), _addr(weight), _addr(scale), _addr(shift),
                        _addr(x_out), _addr(out), _addr(out_scale), None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_norm_residual")


def cb_norm_around(desc: cb_norm_around_desc, x, branch=None, gate=None, after_weight=None, after_bias=None, weight=None,
                   bias=None, scale=None, shift=None, x_out=None, out=None, out_scale=None, stream=None) -> None:
    """The branch, normed after its block, added to ``x`` (into ``x_out``), and the sum normed before the next (into ``out``)."""
    rc = _norm_around(ctypes.addressof(desc), _addr(x), _addr(branch), _addr(gate), _addr(after_weight), _addr(after_bias),
                      _addr(weight), _addr(bias), _addr(scale), _addr(shift), _addr(x_out), _addr(out), _addr(out_scale),
                      None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_norm_around")


def cb_mx_scale_bytes(rows: int, features: int) -> int:
    """Bytes of the scales of ``rows`` rows of ``features`` elements in CB_MXFP4."""
    n = ctypes.c_size_t(0)
    rc = _lib.cb_mx_scale_bytes(rows, features, ctypes.addressof(n))
    if rc < 0:
        _raise(rc, "cb_mx_scale_bytes")
    return n.value


def cb_mx_quantize(desc: cb_mx_desc, x, codes, scales, stream=None) -> None:
    """Rows ``x`` into CB_MXFP4: ``codes`` and ``scales``."""
    rc = _mx_quantize(ctypes.addressof(desc), _addr(x), _addr(codes), _addr(scales), None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_mx_quantize")


def cb_mx_dequantize(desc: cb_mx_desc, codes, scales, x, stream=None) -> None:
    """Rows ``x`` from CB_MXFP4."""
    rc = _mx_dequantize(ctypes.addressof(desc), _addr(codes), _addr(scales), _addr(x), None if stream is None else _stream(stream))
    if rc < 0:
        _raise(rc, "cb_mx_dequantize")


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
