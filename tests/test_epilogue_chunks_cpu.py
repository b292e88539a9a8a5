"""Which warp of a matrix product's epilogue has which chunk of 32 columns of a tile: the kernels' own rules, compiled for the CPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT, HIDDEN, DIRECT, QUANT, HIDDEN_LONG = range(5)
KERNELS = [(OUT, 0), (HIDDEN, 0), (DIRECT, 0), (OUT, 1), (HIDDEN, 1), (DIRECT, 1), (QUANT, 1), (HIDDEN_LONG, 1)]


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    from paper_2608_23429_gb300 import build
    so = str(tmp_path_factory.mktemp("stub") / "libepilogue_stub.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{cuda}", "-o", so, os.path.join(ROOT, "tests", "epilogue_stub.cpp")],
                   check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("results,mx", KERNELS)
@pytest.mark.parametrize("passes", [0, 1])
def test_every_chunk_has_one_warp(stub, results, mx, passes):
    for chunks in range(1, 5 if passes else 7 if mx else 9):
        for tile in range(9):
            assert all(stub.stub_owner(results, mx, passes, tile, c, chunks) >= 0 for c in range(chunks)), (chunks, tile)


@pytest.mark.parametrize("results,mx", KERNELS)
def test_in_passes_a_chunk_has_the_same_warp_in_every_tile(stub, results, mx):
    """The sum of a chunk's passes lies in one place of TMEM, tile after tile: a warp that has no chunk of a tile runs ahead, and would
    write the next tile's first pass there before another has read this one's."""
    for chunks in range(1, 5):
        for c in range(chunks):
            assert len({stub.stub_owner(results, mx, 1, tile, c, chunks) for tile in range(9)}) == 1, (chunks, c)


def test_outputs_in_4_bits_are_dealt_in_turn(stub):
    """In one pass: a tile's three pairs of chunks go to four warps, each of which is without one in turn."""
    free = [{0, 1, 2, 3} - {stub.stub_owner(QUANT, 1, 0, tile, c, 6) for c in range(6)} for tile in range(4)]
    assert all(len(f) == 1 for f in free) and set.union(*free) == {0, 1, 2, 3}
    for tile in range(4):
        assert all(stub.stub_owner(QUANT, 1, 0, tile, c, 6) == stub.stub_owner(QUANT, 1, 0, tile, c + 1, 6) for c in (0, 2, 4))
