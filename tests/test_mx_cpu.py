"""Rows in 4 bits on the CPU: the tests' reference by itself, sizes, and every refusal that comes before a launch."""
import ctypes
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_reference as R  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def test_reference_by_hand():
    v = np.zeros((2, 33))
    v[0, :10] = [6, -5, 5.01, 2.5, 1.75, 0.25, 0.26, -0.74, 3.5, -0.0]  # power 1
    v[0, 32] = 7.0  # power 2: 3.5, a tie
    v[1, 0] = np.inf
    e = R.scale_bytes(v)
    assert e.tolist() == [[127, 128], [255, 0]]
    c = R.codes(v, e)
    assert R.values(c, e, 33)[0, :10].tolist() == [6, -4, 6, 2, 2, 0, 0.5, -0.5, 4, 0]
    assert R.values(c, e, 33)[0, 32] == 8.0 and c[0, 32] == 6 and np.isnan(R.values(c, e, 33)[1, :32]).all()
    assert R.packed(c)[0, :2].tolist() == [7 | 14 << 4, 7 | 4 << 4]
    assert np.array_equal(R.unpacked(R.packed(c)), c)
    assert R.scale_bytes(np.array([[6.99]]))[0, 0] == 127 and R.scale_bytes(np.array([[3.49]]))[0, 0] == 126
    assert R.scale_bytes(np.array([[2.0 ** -149]]))[0, 0] == 0 and R.scale_bytes(np.array([[3.4e38]]))[0, 0] == 253


def test_tiles_by_hand():
    assert [R.place(r, b, 9) for r, b in ((0, 0), (1, 0), (32, 0), (127, 3), (0, 4), (0, 8), (128, 0), (161, 5))] == [
        0, 16, 4, 511, 512, 1024, 1536, 1536 + 512 + 16 + 4 + 1]
    e = np.random.default_rng(0).integers(0, 255, (300, 9)).astype(np.uint8)
    t = R.tiled(e)
    assert t.size == 3 * 3 * 512 and np.array_equal(R.from_tiles(t, 300, 9), e)


def test_scale_bytes(lib):
    block, cb = lib
    for r, k in ((0, 1), (1, 1), (128, 128), (129, 129), (1000, 577)):
        assert block.cb_mx_scale_bytes(r, k) == -(-r // 128) * -(-(-(-k // 32)) // 4) * 512
    for r, k in ((-1, 4), (4, 0), (4, -1)):
        with pytest.raises(cb.CbError) as e:
            block.cb_mx_scale_bytes(r, k)
        assert e.value.status == cb.CB_ERR_ARG
    for r, k in ((1 << 31, 4), (4, 1 << 31)):
        with pytest.raises(cb.CbError) as e:
            block.cb_mx_scale_bytes(r, k)
        assert e.value.status == cb.CB_ERR_LIMIT
    assert cb._lib.cb_mx_scale_bytes(4, 4, None) == cb.CB_ERR_ARG


def test_refusals(lib):
    block, cb = lib
    X, C, S = 0x10000, 0x20000, 0x30000  # never dereferenced
    A, L, M = cb.CB_ERR_ARG, cb.CB_ERR_ALIGN, cb.CB_ERR_LIMIT

    def both(x=X, c=C, s=S, **kw):
        d = dict(rows=4, features=100, dtype=cb.CB_BF16)
        d.update(kw)
        d = block.cb_mx_desc(**d)
        got = set()
        for f, a in ((block.cb_mx_quantize, (x, c, s)), (block.cb_mx_dequantize, (c, s, x))):
            with pytest.raises(cb.CbError) as e:
                f(d, *a)
            got.add(e.value.status)
        assert len(got) == 1
        return got.pop()

    assert both(x=None) == A and both(c=None) == A and both(s=None) == A and both(rows=-1) == A and both(features=0) == A
    assert both(reserved=1) == A and both(dtype=cb.CB_E4M3) == A and both(dtype=cb.CB_MXFP4) == A and both(dtype=-1) == A
    assert both(stride=99) == A and both(stride=-100) == A and both(codes_stride=100) == A and both(codes_stride=96) == A
    assert both(codes_stride=-128) == A and both(codes_stride=130) == A
    assert both(stride=cb.CB_MAX_NUMEL + 1) == M and both(codes_stride=cb.CB_MAX_NUMEL + 32) == M
    assert both(rows=1 << 31) == M and both(features=1 << 31) == M and both(rows=(1 << 31) - 1, features=0x7FFFFF00) == M
    assert both(x=X + 1) == L and both(x=X + 2, dtype=cb.CB_FP32) == L and both(c=C + 8) == L and both(s=S + 8) == L
    for f in (cb._lib.cb_mx_quantize, cb._lib.cb_mx_dequantize):
        assert f(None, X, C, S, None) == A
    nothing = block.cb_mx_desc(rows=0, features=4)
    block.cb_mx_quantize(nothing, None, None, None)
    block.cb_mx_dequantize(nothing, None, None, None)
    assert ctypes.sizeof(block.cb_mx_desc) == 40


def test_linear_refusals(lib):
    block, cb = lib
    A, L, M = cb.CB_ERR_ARG, cb.CB_ERR_ALIGN, cb.CB_ERR_LIMIT
    W, X, O, R_, S, T = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000  # never dereferenced

    def status(f, *a, **kw):
        with pytest.raises(cb.CbError) as e:
            f(*a, **kw)
        return e.value.status

    def create(w=W, n=64, k=100, w_scale=S, **kw):
        return status(block.cb_linear_create, w, n, k, cb.CB_MXFP4, w_scale=w_scale, **kw)

    assert create(w_scale=None) == A and create(w_stride=96) == A and create(w_stride=100) == A and create(w_stride=144) == A
    assert create(w=W + 8) == L and create(w_scale=S + 8) == L and create(w_stride=1 << 33) == M and create(k=(1 << 22) + 1) == M
    layer, wide = block.cb_linear_create(W, 100, 100, cb.CB_MXFP4, w_scale=S), block.cb_linear_create(W, 100, 100, cb.CB_BF16)

    def run(x=X, x_scale=S, resid=None, gate=None, out=O, resid_out=None, layer=layer, **kw):
        d = dict(rows=4, out_dtype=cb.CB_BF16, resid_dtype=cb.CB_BF16, gate_dtype=cb.CB_BF16)
        d.update(kw)
        return status(block.cb_linear_run, layer, block.cb_linear_io(**d), x, x_scale, resid, gate, out, resid_out)

    mx = dict(out_dtype=cb.CB_MXFP4, out_scale=T)
    assert run(x_scale=None) == A and run(x=X + 8) == L and run(x_scale=S + 4) == L and run(x_stride=100) == A and run(x_stride=96) == A
    assert run(x_stride=1 << 33) == M and run(out_dtype=cb.CB_MXFP4) == A and run(out=None, **mx) == A
    assert run(resid=R_, resid_out=R_, **mx) == A and run(out=None, resid=R_, resid_out=R_, **mx) == A
    assert run(out_stride=100, **mx) == A and run(out_stride=96, **mx) == A and run(out=O + 8, **mx) == L
    assert run(out_dtype=cb.CB_MXFP4, out_scale=T + 8) == L and run(out_dtype=cb.CB_E4M3) == A and run(resid_dtype=cb.CB_MXFP4) == A
    assert run(layer=wide, x_scale=None, **mx) == A and run(layer=wide) == A
    block.cb_linear_run(layer, block.cb_linear_io(rows=0), None)
    block.cb_linear_destroy(layer)
    block.cb_linear_destroy(wide)


def test_norm_around_refusals(lib):
    block, cb = lib
    A, L, M = cb.CB_ERR_ARG, cb.CB_ERR_ALIGN, cb.CB_ERR_LIMIT
    P = {n: 0x10000 * (i + 1) for i, n in enumerate(("x", "branch", "gate", "after_weight", "after_bias", "weight", "bias", "scale", "shift",
                                                    "x_out", "out", "out_scale"))}  # never dereferenced
    order = list(P)

    def norm(given=("x", "x_out", "out"), at=None, **kw):
        d = dict(rows=4, hidden=100, tokens=2, x_dtype=cb.CB_BF16, branch_dtype=cb.CB_BF16, param_dtype=cb.CB_BF16, out_dtype=cb.CB_BF16,
                 before=block.CB_NORM_LAYER, before_eps=1e-6)
        d.update(kw)
        a = {**{n: P[n] for n in given}, **(at or {})}
        with pytest.raises(cb.CbError) as e:
            block.cb_norm_around(block.cb_norm_around_desc(**d), *[a.get(n) for n in order])
        return e.value.status

    rms, every = dict(after=block.CB_NORM_RMS), tuple(order[:-1])
    assert norm(("out",)) == A and norm(("x",)) == A and norm(("x", "out", "gate")) == A and norm(("x", "out"), **rms) == A
    assert norm(("x", "branch", "out", "after_weight")) == A and norm(("x", "branch", "out", "after_bias")) == A
    for n in ("weight", "bias"):
        assert norm(("x", "out", n), before=block.CB_NORM_NONE) == A
    for n in ("weight", "bias", "scale", "shift", "out_scale"):
        assert norm(("x", "x_out", n)) == A
    assert norm(("x", "out", "out_scale")) == A and norm(out_dtype=cb.CB_E4M3) == A and norm(out_dtype=cb.CB_MXFP4) == A
    assert norm(("x", "x_out", "out_scale"), out_dtype=cb.CB_MXFP4) == A
    assert norm(rows=-1) == A and norm(hidden=0) == A and norm(tokens=-1) == A and norm(reserved=1) == A
    for n in ("x_dtype", "branch_dtype", "param_dtype"):
        assert norm(**{n: cb.CB_E4M3}) == A and norm(**{n: cb.CB_MXFP4}) == A and norm(**{n: 9}) == A
    assert norm(out_dtype=cb.CB_INT8) == A and norm(after=3) == A and norm(before=-1) == A
    for n in ("after_eps", "before_eps"):
        assert norm(**{n: -1.0}) == A and norm(**{n: float("nan")}) == A and norm(**{n: float("inf")}) == A
    for n in ("x_factor", "branch_factor"):
        assert norm(**{n: float("nan")}) == A and norm(**{n: float("inf")}) == A
    for s in ("x_stride", "branch_stride", "x_out_stride", "out_stride", "line_stride"):
        assert norm(**{s: 99}) == A and norm(**{s: -100}) == A and norm(**{s: cb.CB_MAX_NUMEL + 1}) == M
    mx = dict(given=("x", "out", "out_scale"), out_dtype=cb.CB_MXFP4)
    assert norm(out_stride=100, **mx) == A and norm(out_stride=130, **mx) == A
    assert norm(rows=1 << 31) == M and norm(hidden=1 << 31) == M
    for n in every:
        assert norm(every, {n: P[n] + 1}, **rms) == L
    assert norm(at={"out": P["out"] + 8}, **mx) == L and norm(at={"out_scale": P["out_scale"] + 8}, **mx) == L
    assert norm(("x", "out", "out_scale"), {"out_scale": P["out_scale"] + 2}, out_dtype=cb.CB_E4M3) == L
    assert cb._lib.cb_norm_around(None, *[P["x"]] * 12, None) == A
    block.cb_norm_around(block.cb_norm_around_desc(rows=0, hidden=4), None)
