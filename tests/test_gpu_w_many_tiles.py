"""The operators around a block in 4 bits over more rows and tiles than the GPU works on at once: what a warp or CTA does with the second one and
the next, in every kind of kernel."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_gpu_p_mx_linear as P  # noqa: E402
import test_gpu_q_norm_around as Q  # noqa: E402
import test_gpu_t_mx_passes as T  # noqa: E402
from test_gpu_t_mx_passes import lib  # noqa: E402,F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


# Rows by vectors: warps (up to 1280 elements) and CTAs that have three rows or more each, one behind the other, over the borders of samples; each number of
# chunks a thread, and of warps a row.
@pytest.mark.parametrize("rows,hidden", [(15000, 256), (12000, 512), (8192, 768), (8192, 1024), (8192, 1152), (3000, 2048), (3000, 2560), (3000, 4096),
                                         (1100, 6144), (1100, 8192), (700, 12288), (700, 16384)])
@pytest.mark.parametrize("x,branch", [("bf16", "bf16"), ("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32")])
def test_norms_of_many_rows(lib, rows, hidden, x, branch):  # noqa: F811
    for out, after, before, tokens, param in (("fp32", "layer", "layer", 7, "bf16"), ("e4m3", "rms", "layer", 1, "fp32"), ("bf16", "layer", "rms", 1000, "bf16")):
        Q.check(lib, Q.case(rows, hidden, after, before, x, branch, param, out, tokens=tokens, factors=(1.5, 0.25), inplace=out == "bf16"))


@pytest.mark.parametrize("rows,hidden,x", [(15000, 136, "fp32"), (5000, 1152, "bf16"), (5000, 1160, "fp32"), (3000, 2056, "bf16"), (700, 8192, "fp32")])
def test_norms_of_many_rows_to_4_bits(lib, rows, hidden, x):  # noqa: F811
    """To the bit what cb_mx_quantize makes of the same rows in fp32, which are within the bound of 64 bits."""
    block, cb = lib
    c = Q.case(rows, hidden, "layer", "layer", x, "bf16", out="fp32", tokens=7)
    (h, eh, y, ey), x_out, out, _ = Q.run(lib, c)
    Q.close(out, y, ey, "fp32")
    Q.close(x_out, h, eh, x)
    rows4 = [torch.zeros(rows, -(-hidden // 32) * 16, dtype=torch.uint8, device="cuda"), torch.zeros(block.cb_mx_scale_bytes(rows, hidden), dtype=torch.uint8, device="cuda")]
    block.cb_mx_quantize(block.cb_mx_desc(rows=rows, features=hidden, dtype=cb.CB_FP32), out, *rows4)
    _, again, got, scales = Q.run(lib, {**c, "out": "mx"})
    torch.cuda.synchronize()
    assert torch.equal(again, x_out) and torch.equal(got, rows4[0])
    assert torch.equal(torch.where(scales == 0xA5, 0, scales), torch.where(rows4[1] == 0xA5, 0, rows4[1]))  # (0xA5: a byte that is not written)


@pytest.mark.parametrize("act", ["NONE", "GELU", "SILU"])
@pytest.mark.parametrize("m,n,k", [(4096, 4608, 1152), (6000, 2100, 577), (5000, 1000, 4608), (2600, 4128, 100)])
def test_outputs_in_4_bits_of_many_tiles(lib, m, n, k, act):  # noqa: F811
    """To the bit what cb_mx_quantize makes of the fp32 output, which is within the bound of 64 bits: a bias for each column, tiles of 192 columns
    whose chunks go to the warps in turn."""
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x, xs, xv, xp = T.operand(m, k, g)
    w, ws, wv, wp = T.operand(n, k, g)
    xs, ws = (torch.where((s == 0xFF) | (s == 0), s, s - 4).contiguous() for s in (xs, ws))  # (values of about 1, on both sides of where GELU bends)
    bias = torch.randn(n, generator=g, device="cuda")
    v = (xv @ wv.t()).double() * (xp[:, None] * wp[None, :]).double() / 256 + bias.double()
    e = 4 * U * v.abs() + 4 * U * bias.double().abs()  # (the sums are exact)
    if act != "NONE":
        t = v if act == "SILU" else 1.5957691216057308 * (v + 0.044715 * v ** 3)
        e = 1.2 * e + (8 + 3 * (t.abs().clamp_max(90) + 4)) * U * v.abs()
        v = v / (1 + torch.exp(-t))
    layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws, bias, cb.CB_FP32, getattr(block, "CB_ACT_" + act))
    plain, out, want = torch.empty(m, n, device="cuda"), *(torch.zeros(m, -(-n // 32) * 16, dtype=torch.uint8, device="cuda") for _ in range(2))
    scales, want_scales = (torch.zeros(block.cb_mx_scale_bytes(m, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32), x, xs, out=plain)
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_MXFP4, out_scale=scales.data_ptr()), x, xs, out=out)
    block.cb_mx_quantize(block.cb_mx_desc(rows=m, features=n, dtype=cb.CB_FP32), plain, want, want_scales)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    assert block.cb_linear_device_status() == 0
    P.close(plain, v, e, "fp32")
    assert torch.equal(out, want) and torch.equal(scales, want_scales)


@pytest.mark.parametrize("out,resid", [(None, "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), (None, "fp32"), ("bf16", "fp32"), ("fp32", "fp32"), ("bf16", None), ("fp32", None)])
@pytest.mark.parametrize("m,n,k", [(8192, 1152, 4608), (8192, 1152, 1152), (6000, 2101, 4200), (6000, 2101, 520)])
def test_results_of_many_tiles(lib, m, n, k, out, resid):  # noqa: F811
    """Exact sums, with a bias; hidden states under gates of samples whose rows a warp has several of."""
    T.check(lib, m, n, k, out, resid, gate=resid is not None, tokens=100)
