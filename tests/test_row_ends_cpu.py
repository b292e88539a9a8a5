"""How results leave whose rows start on 16-byte boundaries and end inside one: the host side over the stand-ins of test_block_dispatch_cpu.py."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_block_dispatch_cpu import BF16, DIRECT, FP32, HIDDEN, OUT, library, run, stub  # noqa: E402,F401

E4M3 = 3


@pytest.mark.parametrize("type", [BF16, E4M3])
@pytest.mark.parametrize("kw,results,es", [(dict(out=BF16), OUT, (2,)), (dict(out=FP32), OUT, (4,)), (dict(resid=BF16), HIDDEN, (2,)),
                                           (dict(resid=FP32, out=BF16), HIDDEN, (2, 4))])
@pytest.mark.parametrize("n", [260, 261, 262, 264, 301])
def test_whole_pieces_leave_by_tma(stub, type, kw, results, es, n):  # noqa: F811
    """In bf16 and e4m3; the maps that results leave through end with the last whole piece of 16 bytes."""
    rc, log = run(stub, 300, n, 320, type=type, out_stride=320, resid_stride=320, resid_out_stride=320, **kw)
    assert rc == 0 and log[-1][1]["results"] == results
    wide = [c[1]["wide"] for c in log if c[0] == "map" and c[1]["rows"] == 300]  # x's, and the results'
    whole = n // 8 * 8 if BF16 in kw.values() else n // 4 * 4  # the columns that are whole pieces of all results
    want = [whole * e for e in es] + ([n * (4 if kw["resid"] == FP32 else 2)] if "resid" in kw else [])  # (what is read ends with the row)
    assert sorted(wide) == sorted(want + [320 * (2 if type == BF16 else 1)])


def test_what_the_threads_still_store(stub):  # noqa: F811
    """Rows without a whole piece, and gates whose last piece would be read behind their end."""
    for n, kw in ((7, dict(out=BF16)), (7, dict(out=FP32)), (260, dict(resid=BF16, gate=BF16)), (261, dict(resid=BF16, gate=FP32))):
        stub[0].stub_reset()
        rc, log = run(stub, 300, n, 320, out_stride=264, resid_stride=264, resid_out_stride=264, gate_stride=264, **kw)
        assert rc == 0 and log[-1][1]["results"] == DIRECT, (n, kw)
    stub[0].stub_reset()
    rc, log = run(stub, 300, 260, 320, resid_stride=264, resid_out_stride=264, gate_stride=264, resid=BF16, gate=FP32)
    assert rc == 0 and log[-1][1]["results"] == HIDDEN
