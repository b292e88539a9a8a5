"""Which kernels a process's first products prepare, which loads them onto the device: linear_tc.cu over stand-ins for the CUDA runtime and the kernels."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MX = 256  # numbers of kernels for 4 bits are from here on


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    from paper_2608_23429_gb300 import build
    so = str(tmp_path_factory.mktemp("stub") / "liblaunch_stub.so")
    subprocess.run([build._nvcc(), *build.ARCH, "-std=c++17", "-O1", "-shared", "-cudart", "shared", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    f"-I{build.INCLUDE}", "-o", so, os.path.join(ROOT, "tests", "launch_stub.cpp"), os.path.join(build.CSRC, "linear_tc.cu")], check=True)
    return so


@pytest.fixture()
def stub(library, tmp_path):
    import shutil
    own = str(tmp_path / "launch_stub.so")  # (what is prepared is kept for the process: another copy of the library for each test)
    shutil.copy(library, own)
    lib = ctypes.CDLL(own)
    lib.stub_log.restype = ctypes.c_char_p
    return lib


def log(lib):
    return [(line.split()[0], int(line.split()[-1])) for line in lib.stub_log().decode().splitlines() if line.split()[0] in ("set", "launch")]


def test_products_in_16_and_8_bits_leave_the_kernels_for_4_bits_alone(stub):
    stub.stub_reset(0, -1)
    assert stub.stub_prepare() == 0
    prepared = log(stub)
    assert len(set(prepared)) == 24 and all(k < MX for _, k in prepared)
    assert stub.stub_launch(0, 0, 1) == 0
    assert log(stub)[24:] == [("launch", 1)]


def test_the_first_product_in_4_bits_prepares_its_kernels(stub):
    """On each device, whatever kernel is the first; in a mode in which other streams' captures go on."""
    for device in (0, 3):
        stub.stub_reset(device, -1)
        assert stub.stub_prepare() == 0
        stub.stub_reset(device, -1)
        assert stub.stub_launch(1, 3, 2) == 0
        first = log(stub)
        assert len({k for what, k in first if what == "set"}) == 20 and all(k >= MX for _, k in first) and first[-1][0] == "launch"
        lines = stub.stub_log().decode().splitlines()
        assert lines[0] == "relaxed" and lines[-2] == "as before"
        stub.stub_reset(device, -1)
        assert stub.stub_launch(1, 0, 1) == 0
        assert [what for what, _ in log(stub)] == ["launch"]


def test_a_preparation_that_fails_is_an_error_and_tried_again(stub):
    stub.stub_reset(1, 5)
    assert stub.stub_launch(1, 0, 1) != 0
    assert "launch" not in [what for what, _ in log(stub)] and stub.stub_log().decode().splitlines()[-1] == "as before"
    stub.stub_reset(1, -1)
    assert stub.stub_launch(1, 0, 1) == 0
    assert [what for what, _ in log(stub)] == ["set"] * 20 + ["launch"]
