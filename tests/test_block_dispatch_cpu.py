"""Which kernel a matrix product runs, with what: the host side of cb_linear_* over stand-ins for the CUDA runtime and the launchers
(linear_stub.cpp), on the CPU."""
import ctypes
import os
import re
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT, HIDDEN, DIRECT = 0, 1, 2  # ways in which results leave


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    from paper_2608_23429_gb300 import build
    build.build()
    so = str(tmp_path_factory.mktemp("stub") / "liblinear_stub.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", f"-I{cuda}", "-o", so,
                    os.path.join(ROOT, "tests", "linear_stub.cpp"), "-x", "c++", os.path.join(build.CSRC, "linear.cu")], check=True)
    return so


def _load(path):
    from paper_2608_23429_gb300 import block, chebboost as cb
    lib = ctypes.CDLL(path)
    lib.stub_log.restype = ctypes.c_char_p
    for name in ("cb_linear_create", "cb_linear_run", "cb_linear_destroy", "cb_linear_device_status"):
        getattr(lib, name).argtypes, getattr(lib, name).restype = block._sig[name]
    return lib, block, cb


@pytest.fixture()
def stub(library):
    s = _load(library)
    s[0].stub_reset()
    return s


def _log(lib):
    """(name, {field: value}) of every call noted since the last reset."""
    return [(line.split()[0], {k: int(v) for k, v in re.findall(r"(\w+)=(-?\d+)", line)}) for line in lib.stub_log().decode().splitlines()]


def run(stub, rows, n, k, type=0, out=None, resid=None, gate=None, off=0, **io):
    """One call on addresses that nothing reads; `out`, `resid`, `gate`: their types."""
    lib, block, cb = stub
    d = block.cb_linear_desc(in_features=k, out_features=n, type=type, w=(1 << 40) + off)
    layer = ctypes.c_void_p()
    assert lib.cb_linear_create(ctypes.addressof(d), ctypes.byref(layer)) == 0
    desc = block.cb_linear_io(rows=rows, out_dtype=out or 0, resid_dtype=resid or 0, gate_dtype=gate or 0, **io)
    at = lambda i, t: None if t is None else i << 42  # noqa: E731
    rc = lib.cb_linear_run(layer, ctypes.addressof(desc), (1 << 41) + off, None, at(1, resid), at(2, gate), at(3, out), at(4, resid), None)
    lib.cb_linear_destroy(layer)
    return rc, [c for c in _log(lib) if c[0] != "trim"]


BF16, FP32 = 0, 1


@pytest.mark.parametrize("n,kw,results", [
    ((1 << 29) - 1024, dict(out=FP32), OUT), ((1 << 29) + 64, dict(out=FP32), DIRECT), ((1 << 30) - 1024, dict(out=BF16), OUT),
    ((1 << 30) + 64, dict(out=BF16), DIRECT), ((1 << 29) + 64, dict(resid=FP32), DIRECT), ((1 << 29) + 64, dict(resid=BF16), HIDDEN),
    ((1 << 29) + 64, dict(resid=BF16, gate=FP32), DIRECT), ((1 << 29) + 64, dict(resid=BF16, out=FP32), DIRECT),
    ((1 << 31) - 1024, dict(out=BF16, resid=FP32), DIRECT)])
def test_very_wide_results_leave_by_64_bit_addresses(stub, n, kw, results):
    """The places in a row that copies by TMA are given are signed 32-bit bytes: rows that pass them are stored by the threads."""
    rc, log = run(stub, 33, n, 8, **kw)
    assert rc == 0 and [c[0] for c in log][-1] == "tc"
    assert log[-1][1]["results"] == results
    assert all(c[1]["wide"] < 1 << 31 for c in log if c[0] == "map"), log


def test_parts_of_k_and_operands_off_the_grid(stub):
    assert [c[0] for c in run(stub, 256, 1152, 4608, out=BF16)[1]] == ["malloc", "map", "map", "map", "tc", "join", "free"]
    stub[0].stub_reset()
    assert [c[0] for c in run(stub, 4096, 1152, 1152, off=2, out=BF16)[1]] == ["malloc", "pack", "map", "map", "map", "tc", "free"]
    stub[0].stub_reset()
    assert [c[0] for c in run(stub, 32, 1152, 4608, out=BF16)[1]] == ["few"]


def test_the_last_layer_gives_the_workspace_back(stub):
    lib, block, cb = stub
    run(stub, 4096, 1152, 1152, off=2, out=BF16)  # the pool exists from here on
    layers = [ctypes.c_void_p() for _ in range(3)]
    d = block.cb_linear_desc(in_features=64, out_features=64, w=1 << 40)
    for l in layers:
        assert lib.cb_linear_create(ctypes.addressof(d), ctypes.byref(l)) == 0
    lib.stub_reset()
    lib.cb_linear_destroy(None)
    lib.cb_linear_destroy(layers[1])
    lib.cb_linear_destroy(layers[0])
    assert _log(lib) == []
    lib.cb_linear_destroy(layers[2])
    assert [c[0] for c in _log(lib)] == ["trim"]


def test_the_status_is_taken_and_cleared_in_one_step(stub):
    """A code that another stream's product notes between a read and a clearing would be lost: one kernel exchanges the word."""
    lib = stub[0]
    status = ctypes.c_int(-1)
    assert lib.cb_linear_device_status(ctypes.addressof(status), None) == 0 and status.value == 0
    assert [c[0] for c in _log(lib)] == ["malloc", "take_status", "memcpy", "free", "synchronize"]
    for fails in ("malloc", "take_status", "memcpy", "free", "synchronize"):
        lib.stub_reset()
        lib.stub_fail(fails.encode())
        status.value = -1
        assert lib.cb_linear_device_status(ctypes.addressof(status), None) == -7 and status.value == -1
        names = [c[0] for c in _log(lib)]
        assert fails == "malloc" or "free" in names  # the word that it was taken to is given back


NO_PAIRS = """
import sys
sys.path.insert(0, {tests!r})
import test_block_dispatch_cpu as t
stub = t._load({so!r})
stub[0].stub_pairs(0)
for m, n, k in ((33, 64, 64), (4096, 1152, 1152), (256, 1152, 4608)):
    stub[0].stub_reset()
    rc, log = t.run(stub, m, n, k, out=0)
    tc = [f for name, f in log if name == "tc"]
    assert rc == 0 and [f["cg"] for f in tc] == [1] and tc[0]["grid"] > 0, log
"""


def test_no_room_for_pairs_of_ctas(library):
    """A device (or its share of one) on which no two CTAs can run as a pair: single ones, and no division by their number."""
    r = subprocess.run([sys.executable, "-c", NO_PAIRS.format(tests=os.path.join(ROOT, "tests"), so=library)], cwd=ROOT,
                       capture_output=True, text=True, timeout=200)
    assert r.returncode == 0, (r.returncode, r.stderr)


def test_each_device_status_is_a_bit_of_its_own():
    """...and every code that a kernel notes without having waited says so."""
    from paper_2608_23429_gb300 import build, chebboost as cb
    header = open(os.path.join(ROOT, "include", "chebboost.h")).read()
    codes = {name: int(v) for name, v in re.findall(r"\b(CB_DEV_\w+) = (\d+)", header)}
    assert len(codes) >= 4 and sorted(codes.values()) == [1 << i for i in range(len(codes))]
    assert all(getattr(cb, name) == v for name, v in codes.items())
    kernel = open(os.path.join(build.CSRC, "linear_tc.cuh")).read()
    assert re.findall(r"record\(A\.status, (\w+)\)", kernel) == ["CB_DEV_PLACEMENT"]
