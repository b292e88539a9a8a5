"""The device memory that cb_linear_run keeps between calls."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

GIVEN_BACK = """
import torch
from paper_2608_23429_gb300 import block, chebboost as cb
n, k = 8192, 16383  # 268 MB of weights off the grid, copied for each call
x, w = torch.ones(64, k, device="cuda").bfloat16(), torch.ones(n, k, device="cuda").bfloat16()
y = torch.empty(64, n, device="cuda").bfloat16()
io = block.cb_linear_io(rows=64, out_dtype=cb.CB_BF16)
def free():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]
first = [block.cb_linear_create(w, n, k, cb.CB_BF16) for _ in range(2)]
few = block.cb_linear_io(rows=1, out_dtype=cb.CB_BF16)
block.cb_linear_run(first[0], few, x, out=y)  # the modules are loaded
before = free()
for turn in range(2):
    block.cb_linear_run(first[0], io, x, out=y)
    held = before - free()
    assert held > 200e6, held
block.cb_linear_destroy(first[0])
assert before - free() > 200e6
block.cb_linear_destroy(first[1])
assert before - free() < 64e6, before - free()
layer = block.cb_linear_create(w, n, k, cb.CB_BF16)
block.cb_linear_run(layer, io, x, out=y)
torch.cuda.synchronize()
assert bool((y == torch.tensor(float(k)).bfloat16().item()).all())
block.cb_linear_destroy(layer)
"""


def test_memory_is_given_back_with_the_last_layer():
    """In a process of its own, which nothing else takes memory in. (Other processes of the device would be noticed, too: a margin of 64 MB.)"""
    from paper_2608_23429_gb300 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", GIVEN_BACK], cwd=Path(__file__).parents[1], capture_output=True, text=True, timeout=200)
    assert r.returncode == 0, r.stderr
