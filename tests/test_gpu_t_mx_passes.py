"""cb_linear_run in 4 bits over sums that are taken in passes, in several tiles a CTA: partial sums wait in TMEM for the next pass.

Sums are exact, so results are compared to the bit: codes of magnitudes up to 2 are halves, the products quarters, and 66000 of them at most 4 stay
below 2^20 quarters; every row of x and of w has one power of two of its own, biases are quarters of that size, hidden states and gates such that the sum
fits 24 bits."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def operand(rows, k, g):
    """(codes, scales as they lie in memory, values without the rows' powers of two, these powers)."""
    blocks = -(-k // 32)
    c = torch.randint(0, 5, (rows, blocks * 32), generator=g, device="cuda", dtype=torch.uint8)  # 0, 1/2, 1, 3/2, 2
    c |= torch.randint(0, 2, c.shape, generator=g, device="cuda", dtype=torch.uint8) << 3
    c[:, k:] = 0
    e = torch.randint(125, 130, (rows,), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.from_numpy(R.tiled(np.repeat(e.cpu().numpy()[:, None], blocks, 1), 0xFF)).cuda()
    v = (c[:, :k] & 7).float() * 0.5
    v = torch.where(c[:, :k] >= 8, -v, v)
    return c[:, 0::2] | c[:, 1::2] << 4, scales, v, torch.exp2(e.float() - 127)


def check(lib, m, n, k, out, resid=None, gate=False, tokens=0):
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "mx": cb.CB_MXFP4, None: cb.CB_BF16}
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda").float()  # noqa: E731
    x, xs, xv, xp = operand(m, k, g)
    w, ws, wv, wp = operand(n, k, g)
    bias = ints(-400, 401, n) / 16
    want = (xv @ wv.t()) * xp[:, None] * wp[None, :] + bias
    y = {None: None, "mx": None}.get(out, torch.full((m, n), 7.0, device="cuda").to(DT.get(out, torch.float32)))
    scales = None
    if out == "mx":
        y = torch.full((m, -(-n // 32) * 16), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((block.cb_mx_scale_bytes(m, n),), 0xA5, dtype=torch.uint8, device="cuda")
    r = gates = xo = None
    if resid:
        r = (ints(-64, 65, m, n) / 4).to(DT[resid])
        xo = torch.empty_like(r)
        samples = -(-m // tokens) if tokens else 1
        gates = torch.exp2(ints(-1, 2, samples, n)) if gate else None
    layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws, bias, cb.CB_FP32)
    io = block.cb_linear_io(rows=m, tokens=tokens, out_dtype=code[out], resid_dtype=code[resid], gate_dtype=cb.CB_FP32,
                            out_scale=None if scales is None else scales.data_ptr())
    for _ in range(3):
        block.cb_linear_run(layer, io, x, xs, r, gates, y, xo)
        torch.cuda.synchronize()
        assert block.cb_linear_device_status() == 0
        if out == "mx":
            R.check_quantised(want.double().cpu().numpy(), np.zeros((m, n)), y.cpu().numpy(), scales.cpu().numpy())
        elif out:
            assert torch.equal(y, want.to(DT[out])), int((y != want.to(DT[out])).sum())
        if resid:
            h = want if gates is None else want * gates[torch.arange(m, device="cuda") // (tokens or m)]
            h = (h + r.float()).to(DT[resid])
            assert torch.equal(xo, h), int((xo != h).sum())
    block.cb_linear_destroy(layer)


@pytest.mark.parametrize("m,n,k", [(2600, 2600, 66000), (3000, 1000, 131328), (5000, 2320, 16416), (3000, 2304, 40000)])
def test_outputs_in_4_bits(lib, m, n, k):
    """In passes, where half of the warps have no chunk of a tile; and in one pass over the longer sums that have only one."""
    check(lib, m, n, k, "mx")


# (sizes whose way test_mx_passes_cpu.py tells: passes, and more tiles than CTAs)
@pytest.mark.parametrize("m,n,k,out,resid", [
    (6000, 2100, 16640, "fp32", None), (6000, 2100, 40000, "fp32", None),  # results by TMA
    (6000, 2100, 16640, None, "fp32"), (4000, 2100, 33000, "fp32", "fp32"), (4000, 2100, 33000, "bf16", "fp32"),  # hidden states
    (4000, 2101, 16640, "fp32", None), (4000, 2101, 33000, "bf16", "fp32"),  # by the threads
    (4000, 2104, 66000, "bf16", None), (4000, 2104, 66000, "bf16", "bf16"), (3000, 2101, 66000, None, "bf16")])
def test_results_of_every_kind(lib, m, n, k, out, resid):
    check(lib, m, n, k, out, resid, gate=resid is not None, tokens=100)
