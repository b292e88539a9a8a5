"""Which kernel a product in 4 bits runs, with what: the host side over the stand-ins of test_block_dispatch_cpu.py."""
import ctypes
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_block_dispatch_cpu import _load, _log, library  # noqa: E402,F401

OUT, HIDDEN, DIRECT, QUANT, HIDDEN_LONG = range(5)
BF16, FP32, MX = 0, 1, 4


@pytest.fixture()
def stub(library):  # noqa: F811
    s = _load(library)
    s[0].stub_reset()
    return s


def run(stub, rows, n, k, out=None, resid=None, gate=None, **io):
    """One call on addresses that nothing reads; `out`, `resid`, `gate`: their types."""
    lib, block, cb = stub
    d = block.cb_linear_desc(in_features=k, out_features=n, type=cb.CB_MXFP4, w=1 << 40, w_scale=(1 << 40) + (1 << 38))
    layer = ctypes.c_void_p()
    assert lib.cb_linear_create(ctypes.addressof(d), ctypes.byref(layer)) == 0
    desc = block.cb_linear_io(rows=rows, out_dtype=out or 0, resid_dtype=resid or 0, gate_dtype=gate or 0, out_scale=1 << 46, **io)
    at = lambda i, t: None if t is None else i << 42  # noqa: E731
    rc = lib.cb_linear_run(layer, ctypes.addressof(desc), 1 << 41, (1 << 41) + (1 << 38), at(1, resid), at(2, gate), at(3, out), at(4, resid), None)
    lib.cb_linear_destroy(layer)
    return rc, [c for c in _log(lib) if c[0] != "trim"]


@pytest.mark.parametrize("rows,n,k,kw,results", [
    (1, 6912, 1152, dict(out=BF16), OUT), (4096, 4608, 1152, dict(out=FP32), OUT), (4096, 4608, 1152, dict(out=MX), QUANT), (8, 33, 40, dict(out=MX), QUANT),
    (4096, 1152, 4096, dict(resid=BF16, gate=BF16), HIDDEN), (4096, 1152, 4097, dict(resid=FP32, out=BF16), HIDDEN_LONG),
    (999, 1155, 577, dict(resid=FP32, out=BF16), DIRECT), (999, 1155, 577, dict(out=BF16), DIRECT)])
def test_how_results_leave(stub, rows, n, k, kw, results):
    rc, log = run(stub, rows, n, k, **kw)
    assert rc == 0 and log[-1][0] == "tc" and log[-1][1]["results"] == results
    f = log[-1][1]
    assert f["tile_n"] % 64 == 0 and 64 <= f["tile_n"] <= 192 and f["parts"] == 1 and f["fp8"] == 0
    maps = [c[1] for c in log if c[0] == "map"]
    blocks = -(-k // 32)
    codes = [m for m in maps if m["wide"] == 16 * blocks]
    assert {m["rows"] for m in codes} == {rows, n} and all(m["stride"] == 16 * blocks for m in codes)
    tiles = -(-blocks // 4)
    assert [(m["rows"], m["stride"]) for m in maps if m["wide"] == 128 * tiles and m["stride"] == 512 * tiles][:2] == [
        (-(-rows // 128), 512 * tiles), (-(-n // 128), 512 * tiles)]


def test_long_sums(stub):
    """fp32 results in passes of 16384 features, in tiles of 128 columns at most; results in 4 bits are not split over K."""
    f = run(stub, 4096, 4096, 16384, out=FP32)[1][-1][1]
    assert f["passes"] == 1 and f["tile_n"] == 192
    stub[0].stub_reset()
    f = run(stub, 4096, 4096, 16416, out=FP32)[1][-1][1]
    assert f["passes"] == 2 and f["tile_n"] <= 128
    stub[0].stub_reset()
    assert [c[0] for c in run(stub, 256, 128, 32768, out=BF16)[1] if c[0] != "map"] == ["malloc", "tc", "join", "free"]
    stub[0].stub_reset()
    assert [c[0] for c in run(stub, 256, 128, 32768, out=MX)[1] if c[0] != "map"] == ["tc"]


def test_failures_leave_nothing_behind(stub):
    lib = stub[0]
    for fails in ("malloc", "tc", "join", "free"):
        lib.stub_reset()
        lib.stub_fail(fails.encode())
        rc, log = run(stub, 256, 128, 32768, out=BF16)
        assert rc == -7 and (fails == "malloc") == ("free" not in [c[0] for c in log])


def test_rows_that_end_inside_16_bytes_are_stored_by_the_threads(stub):
    """A copy by TMA would write the rest of the piece, too."""
    for kw, results in ((dict(out=BF16), OUT), (dict(resid=BF16), HIDDEN), (dict(resid=FP32, out=BF16), HIDDEN)):
        for n, off in ((264, False), (260, True), (262, True)):
            stub[0].stub_reset()
            rc, log = run(stub, 300, n, 320, out_stride=264, resid_stride=264, resid_out_stride=264, gate_stride=264, **kw)
            assert rc == 0 and log[-1][1]["results"] == (DIRECT if off else results), (n, kw)


@pytest.mark.parametrize("out", [None, BF16, FP32, MX])
@pytest.mark.parametrize("resid", [None, BF16, FP32])
def test_every_size_is_served(stub, out, resid):
    """No choice of tiles leaves a kernel without shared memory for its stages."""
    if (out is None and resid is None) or (out == MX and resid is not None):
        return
    lib = stub[0]
    for rows in (1, 8, 40, 129, 300, 1000, 4096, 8192, 30000):
        for n in (8, 64, 200, 1152, 4608, 12288):
            for k in (32, 1152, 4096, 4608, 16384, 40000):
                lib.stub_reset()
                rc, log = run(stub, rows, n, k, out=out, resid=resid, gate=resid)
                assert rc == 0 and "tc" in [c[0] for c in log], (rows, n, k)
