"""The full step's operators on the CPU: exported symbols and every refusal that comes before a launch."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def _header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "chebboost_block.h")).read(), flags=re.S)


def test_every_declared_symbol_is_bound(lib):
    block, cb = lib
    names = set(re.findall(r"\bint (cb_\w+)\s*\(", _header())) | set(re.findall(r"\bvoid (cb_\w+)\s*\(", _header()))
    assert names == set(block.EXPORTED)
    so = ctypes.CDLL(cb.LIB_PATH)
    assert all(hasattr(so, n) for n in names)


def test_constants_and_structs_match_the_header(lib):
    block, cb = lib
    for name, value in re.findall(r"\b(CB_ACT_\w+)\s*=\s*(-?\d+)", _header()):
        assert getattr(block, name) == int(value), name
    for name, value in re.findall(r"#define (CB_\w+) \(1LL << (\d+)\)", _header()):
        assert getattr(block, name) == 1 << int(value), name
    for body, name in re.findall(r"typedef struct \{(.*?)\}\s*(cb_\w+);", _header(), flags=re.S):
        fields = re.findall(r"(\w+)\s*;", body)
        assert fields == [f for f, _ in getattr(block, name)._fields_], name


def _status(cb, f, *a, **kw):
    with pytest.raises(cb.CbError) as e:
        f(*a, **kw)
    return e.value.status


def test_norm_refusals(lib):
    block, cb = lib
    X, B, G, O, S = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000  # never dereferenced

    def norm(x=X, branch=None, gate=None, weight=None, scale=None, shift=None, x_out=None, out=O, out_scale=None, **kw):
        d = dict(rows=4, hidden=64, tokens=2, x_dtype=cb.CB_BF16, branch_dtype=cb.CB_BF16, param_dtype=cb.CB_BF16,
                 out_dtype=cb.CB_BF16, eps=1e-6)
        d.update(kw)
        return _status(cb, block.cb_norm_residual, block.cb_norm_desc(**d), x, branch, gate, weight, scale, shift, x_out,
                       out, out_scale)

    A, L, M = cb.CB_ERR_ARG, cb.CB_ERR_ALIGN, cb.CB_ERR_LIMIT
    assert norm(x=None) == A and norm(out=None) == A and norm(gate=G) == A
    assert norm(rows=-1) == A and norm(hidden=0) == A and norm(tokens=-1) == A and norm(reserved=1) == A
    assert norm(x_dtype=cb.CB_E4M3) == A and norm(branch_dtype=cb.CB_INT8) == A and norm(param_dtype=7) == A
    assert norm(out_dtype=cb.CB_INT8) == A and norm(out_dtype=-1) == A
    assert norm(out_dtype=cb.CB_E4M3) == A and norm(out_scale=S) == A
    assert norm(eps=-1.0) == A and norm(eps=float("nan")) == A and norm(eps=float("inf")) == A
    for s in ("x_stride", "branch_stride", "x_out_stride", "out_stride", "line_stride"):
        assert norm(**{s: 63}) == A and norm(**{s: -64}) == A and norm(**{s: cb.CB_MAX_NUMEL + 1}) == M
    assert norm(rows=1 << 31) == M and norm(hidden=1 << 31) == M
    for p in ("x", "branch", "weight", "scale", "shift", "x_out", "out"):
        assert norm(**{p: 0x10001}) == L
    assert norm(branch=B, gate=G + 1) == L
    assert norm(x=X + 2, x_dtype=cb.CB_FP32) == L and norm(out_dtype=cb.CB_E4M3, out_scale=S + 2) == L
    assert cb._lib.cb_norm_residual(None, X, None, None, None, None, None, None, O, None, None) == A


def test_linear_refusals(lib):
    block, cb = lib
    A, L, M = cb.CB_ERR_ARG, cb.CB_ERR_ALIGN, cb.CB_ERR_LIMIT
    W, X, O, R, G, S = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000  # never dereferenced

    def create(w=W, n=64, k=64, type=cb.CB_BF16, **kw):
        return _status(cb, block.cb_linear_create, w, n, k, type, **kw)

    assert create(w=None) == A and create(n=0) == A and create(k=0) == A and create(k=-5) == A
    assert create(type=cb.CB_FP32) == A and create(type=cb.CB_INT8) == A and create(type=9) == A
    assert create(bias=W, bias_dtype=cb.CB_E4M3) == A and create(activation=3) == A and create(activation=-1) == A
    assert create(w_scale=S) == A and create(w_stride=63) == A and create(w_stride=-64) == A
    assert create(n=1 << 31) == M and create(k=1 << 31) == M and create(w_stride=1 << 31) == M
    assert create(w=W + 1) == L and create(bias=W + 1) == L and create(bias=W + 2, bias_dtype=cb.CB_FP32) == L
    assert create(type=cb.CB_E4M3, w_scale=S + 2) == L

    layers = {t: block.cb_linear_create(W, 64, 64, t) for t in (cb.CB_BF16, cb.CB_E4M3)}

    def run(x=X, x_scale=None, resid=None, gate=None, out=O, resid_out=None, type=cb.CB_BF16, **kw):
        d = dict(rows=4, out_dtype=cb.CB_BF16, resid_dtype=cb.CB_BF16, gate_dtype=cb.CB_BF16)
        d.update(kw)
        return _status(cb, block.cb_linear_run, layers[type], block.cb_linear_io(**d), x, x_scale, resid, gate, out, resid_out)

    assert run(x=None) == A and run(out=None) == A and run(resid=R) == A and run(resid_out=R) == A and run(gate=G) == A
    assert run(x_scale=S) == A and run(rows=-1) == A and run(tokens=-1) == A and run(reserved=1) == A
    for t in ("out_dtype", "resid_dtype", "gate_dtype"):
        assert run(**{t: cb.CB_E4M3}) == A and run(**{t: cb.CB_INT8}) == A and run(**{t: -1}) == A
    for s in ("x_stride", "out_stride", "resid_stride", "resid_out_stride", "gate_stride"):
        assert run(**{s: 63}) == A and run(**{s: -64}) == A and run(**{s: cb.CB_MAX_NUMEL + 1}) == M
    assert run(rows=1 << 31) == M
    assert run(x=X + 1) == L and run(out=O + 1) == L and run(resid=R + 1, resid_out=R) == L
    assert run(resid=R, resid_out=R, gate=G + 1) == L and run(x_scale=S + 1, type=cb.CB_E4M3) == L
    assert run(out=O + 2, out_dtype=cb.CB_FP32) == L
    block.cb_linear_run(layers[cb.CB_BF16], block.cb_linear_io(rows=0), None)  # no rows: nothing to do
    for layer in layers.values():
        block.cb_linear_destroy(layer)
    assert cb._lib.cb_linear_run(None, None, X, None, None, None, O, None, None) == A
    assert cb._lib.cb_linear_create(None, ctypes.byref(ctypes.c_void_p())) == A
    assert cb._lib.cb_linear_device_status(None, None) == A
    block.cb_linear_destroy(None)
