"""A process's first product in 4 bits, which prepares its kernels, in a graph that is being captured; with and without a product in bf16 before it."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys, torch
from paper_2608_23429_gb300 import block, chebboost as cb, mlp_branch as M
x, w = torch.randint(-2, 3, (300, 64), device="cuda").float(), torch.randint(-2, 3, (264, 64), device="cuda").float()
x[:, ::32], w[:, ::32] = 2.0, 2.0  # whole numbers under a power of two of 1/2: exact
if sys.argv[1] == "after":
    y, xb, wb = torch.empty(300, 264, device="cuda"), x.bfloat16(), w.bfloat16()
    layer = block.cb_linear_create(wb, 264, 64, cb.CB_BF16)
    block.cb_linear_run(layer, block.cb_linear_io(rows=300, out_dtype=cb.CB_FP32), xb, out=y)
    torch.cuda.synchronize()
    assert torch.equal(y, x @ w.t())
held, wh = M.quantised(x), M.quantised(w)
layer = block.cb_linear_create(wh[0], 264, 64, cb.CB_MXFP4, wh[1])
out = torch.zeros(300, 264, device="cuda")
io = block.cb_linear_io(rows=300, out_dtype=cb.CB_FP32)
torch.cuda.synchronize()
s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=s):
    block.cb_linear_run(layer, io, *held, out=out, stream=s)
for _ in range(2):
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, x @ w.t())
assert block.cb_linear_device_status() == 0
block.cb_linear_destroy(layer)
print("as it should be")
"""


@pytest.mark.parametrize("when", ["first", "after"])
def test_a_captured_first_product_in_4_bits(when):
    from paper_2608_23429_gb300 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", PROGRAM, when], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "as it should be" in r.stdout, r.stdout + r.stderr
