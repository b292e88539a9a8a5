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
