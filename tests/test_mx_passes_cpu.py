"""Over how many passes a product in 4 bits sums K, and in tiles of how many columns: the host side over the stand-ins of test_block_dispatch_cpu.py."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_block_dispatch_cpu import library  # noqa: E402,F401
from test_mx_dispatch_cpu import BF16, FP32, MX, QUANT, run, stub  # noqa: E402,F401


@pytest.mark.parametrize("k", [16384, 16416, 40000, 65536])
def test_outputs_in_4_bits_are_no_fp32_results(stub, k):  # noqa: F811
    """What passes save of a sum is lost in the rounding to 4 bits, up to the length from which bf16 results have them too."""
    f = run(stub, 4096, 4608, k, out=MX)[1][-1][1]
    assert f["results"] == QUANT and f["passes"] == 1 and f["tile_n"] == 192


def test_longer_sums_have_passes(stub):  # noqa: F811
    for out in (MX, BF16):
        stub[0].stub_reset()
        f = run(stub, 4096, 4608, 65568, out=out)[1][-1][1]
        assert f["passes"] == 9 and f["tile_n"] == 128


@pytest.mark.parametrize("m,n,k,out,resid", [
    (6000, 2100, 16640, FP32, None), (6000, 2100, 40000, FP32, None), (6000, 2100, 16640, None, FP32), (4000, 2100, 33000, FP32, FP32),
    (4000, 2100, 33000, BF16, FP32), (4000, 2101, 16640, FP32, None), (4000, 2101, 33000, BF16, FP32), (4000, 2104, 66000, BF16, None),
    (4000, 2104, 66000, BF16, BF16), (3000, 2101, 66000, None, BF16), (2600, 2600, 66000, MX, None), (3000, 1000, 131328, MX, None)])
def test_the_sizes_of_the_tests_on_a_gpu_have_passes(stub, m, n, k, out, resid):  # noqa: F811
    """test_gpu_t_mx_passes.py: and several tiles for a CTA, or a pair of them (but the last)."""
    f = run(stub, m, n, k, out=out, resid=resid, gate=None if resid is None else FP32)[1][-1][1]
    tiles = -(-m // (128 * f["cg"])) * -(-n // f["tile_n"])
    assert f["passes"] > 1 and f["parts"] == 1 and (tiles > f["grid"] // f["cg"] or (m, n) == (3000, 1000)), (f, tiles)
