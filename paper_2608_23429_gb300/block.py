"""ctypes binding of the full step's operators (``include/chebboost_block.h``), same names, marshalling only.

The operators live in libchebboost with the rest; pointers, streams, errors and
constants are those of :mod:`paper_2608_23429_gb300.chebboost`.
"""
from __future__ import annotations

import ctypes

from .chebboost import _addr, _check, _lib, _stream

_P, _I, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64


class cb_norm_desc(ctypes.Structure):
    """Sizes and types of :func:`cb_norm_residual`; strides of 0 mean contiguous."""
    _fields_ = [("rows", _L), ("hidden", _L), ("tokens", _L), ("x_stride", _L), ("branch_stride", _L),
                ("x_out_stride", _L), ("out_stride", _L), ("line_stride", _L), ("x_dtype", _I), ("branch_dtype", _I),
                ("param_dtype", _I), ("out_dtype", _I), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


_sig = {
    "cb_norm_residual": ([_P] * 11, _I),
}
for _name, (_args, _res) in _sig.items():
    _f = getattr(_lib, _name)
    _f.argtypes, _f.restype = _args, _res

EXPORTED = tuple(_sig)


def cb_norm_residual(desc: cb_norm_desc, x, branch=None, gate=None, weight=None, scale=None, shift=None, x_out=None,
                     out=None, out_scale=None, stream=None) -> None:
    """RMS norm of ``x + gate * branch`` into ``out`` (with ``out_scale`` where it is e4m3), the sum into ``x_out``."""
    _check(_lib.cb_norm_residual(ctypes.addressof(desc), _addr(x), _addr(branch), _addr(gate), _addr(weight),
                                 _addr(scale), _addr(shift), _addr(x_out), _addr(out), _addr(out_scale),
                                 _stream(stream)), "cb_norm_residual")
