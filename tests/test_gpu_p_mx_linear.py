"""cb_linear_run with rows and weights in 4 bits, against plain arithmetic in 64 bits on the values that the codes stand for.

Bounds (u = 2^-24): products of codes and of their powers of two are exact in fp32, so a sum of K of them is off by (K + 1) u sum_k
|x w| at most in any order; bias, activation and hidden state as for other operands (test_gpu_g_linear.py). An output in 4 bits is what
the format makes of some value within that bound: its scale lies between those of the block's largest magnitude less and more the bound, and each
code between those of the value less and more the bound, under that scale."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def half_step(v, dtype):
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -126)))
    return torch.exp2(e - (8 if dtype == "bf16" else 24))


def close(got, want, slack, dtype):
    err = (got.double() - want).abs()
    bad = ~(err <= slack + half_step(want.abs() + slack, dtype))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist(), float(err.max()))


def operand(v, pad_blocks=0):
    """Rows in 4 bits as they lie in memory (with 255 for rows behind the last), their values on the GPU, and their stride."""
    held, codes, _ = R.quantised(v)
    r, wide = codes.shape[0], codes.shape[1] + 16 * pad_blocks
    c = np.full((r, wide), 0xFF, np.uint8)
    c[:, :codes.shape[1]] = codes
    return torch.from_numpy(c).cuda(), torch.from_numpy(R.tiled(R.scale_bytes(v), 0xFF)).cuda(), torch.from_numpy(held).cuda(), 2 * wide


def rows_of(rows, n, pad, off, dtype, fill):
    buf = torch.zeros(off + rows * (n + pad) + 16, dtype=DT[dtype], device="cuda")
    v = buf[off:off + rows * (n + pad)].view(rows, n + pad)[:, :n]
    v.copy_(fill)
    return v


def case(m, n, k, act="NONE", out="bf16", resid=None, gate=None, bias="bf16", tokens=0, pad=0, off=0, xpad=0, inplace=False):
    return dict(m=m, n=n, k=k, act=act, out=out, resid=resid, gate=gate, bias=bias, tokens=tokens, pad=pad, off=off, xpad=xpad, inplace=inplace)


def run(lib, c, seed=0, stream=None, spread=0.5):
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "mx": cb.CB_MXFP4, None: cb.CB_BF16}
    rng = np.random.default_rng(seed + c["m"] + c["n"])
    g = torch.Generator(device="cuda").manual_seed(seed + c["k"])
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    m, n, k = c["m"], c["n"], c["k"]
    x, xs, xv, x_stride = operand((rng.standard_normal((m, k)) + 0.1) * np.exp(spread * rng.standard_normal((m, 1))), c["xpad"])
    w, ws, wv, w_stride = operand(rng.standard_normal((n, k)) / k ** 0.5 * np.exp(spread * rng.standard_normal((1, k))), c["xpad"])
    samples = -(-m // c["tokens"]) if c["tokens"] else 1
    line = lambda rows, t, s: rows_of(rows, n, c["pad"], c["off"], t, s * r(rows, n))  # noqa: E731
    bias = line(1, c["bias"], 0.3) if c["bias"] else None
    resid = line(m, c["resid"], 1.0) if c["resid"] else None
    gate = line(samples, c["gate"], 1.0) if c["gate"] else None
    # expected: (v, its bound), (hidden state, its bound before rounding)
    v, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias is not None:
        v, size = v + bias.double(), size + bias.double().abs()
    e = (k + 4) * U * size
    if c["act"] != "NONE":
        t = v if c["act"] == "SILU" else 1.5957691216057308 * (v + 0.044715 * v ** 3)
        e = 1.2 * e + (8 + 3 * (t.abs().clamp_max(90) + 4)) * U * v.abs()
        v = v / (1 + torch.exp(-t))
    h = eh = xo = out = out_scale = None
    if resid is not None:
        gg = torch.ones((), dtype=torch.float64, device="cuda")
        if gate is not None:
            gg = gate.double()[torch.arange(m, device="cuda") // (c["tokens"] or m)]
        h, eh = resid.double() + gg * v, gg.abs() * e + 1.01 * U * (resid.double().abs() + (gg * v).abs())
        xo = resid if c["inplace"] else rows_of(m, n, c["pad"], c["off"], c["resid"], torch.zeros((), device="cuda"))
    n_stride = n + c["pad"]
    out_stride = n_stride
    if c["out"] == "mx":
        out_stride = -(-n // 32) * 32 + 32 * c["xpad"]
        out = torch.full((m, out_stride // 2), 0xA5, dtype=torch.uint8, device="cuda")
        out_scale = torch.full((block.cb_mx_scale_bytes(m, n),), 0xA5, dtype=torch.uint8, device="cuda")
    elif c["out"]:
        out = rows_of(m, n, c["pad"], c["off"], c["out"], torch.full((), 7.0, device="cuda"))
    layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws, bias, code[c["bias"]], getattr(block, "CB_ACT_" + c["act"]), w_stride=w_stride)
    io = block.cb_linear_io(rows=m, tokens=c["tokens"], x_stride=x_stride, out_stride=out_stride, resid_stride=n_stride,
                            resid_out_stride=n_stride, gate_stride=n_stride, out_dtype=code[c["out"]], resid_dtype=code[c["resid"]],
                            gate_dtype=code[c["gate"]], out_scale=None if out_scale is None else out_scale.data_ptr())
    torch.cuda.synchronize()
    block.cb_linear_run(layer, io, x, xs, resid, gate, out, xo, stream)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    return (v, e, h, eh), out, xo, out_scale


def check(lib, c, seed=0, **kw):
    (v, e, h, eh), out, xo, scales = run(lib, c, seed, **kw)
    assert lib[0].cb_linear_device_status() == 0
    if c["out"] == "mx":
        R.check_quantised(v.cpu().numpy(), e.cpu().numpy(), out.cpu().numpy(), scales.cpu().numpy())
    elif out is not None:
        close(out, v, e, c["out"])
    if xo is not None:
        close(xo, h, eh, c["resid"])
    for t in (out, xo):  # what lies between rows stays as it was
        if t is not None and t.dtype != torch.uint8 and c["pad"] and not c["inplace"]:
            whole = torch.as_strided(t, (c["m"], c["n"] + c["pad"]), (c["n"] + c["pad"], 1), t.storage_offset())
            assert float(whole[:, c["n"]:].abs().max()) == 0.0


CASES = [
    # one tile; then a whole one of each width, the second half of a tile of scales, more rows
    case(128, 64, 64, out="fp32", bias=None), case(128, 64, 128, out="fp32"), case(128, 64, 256, out="fp32"), case(128, 64, 512, out="fp32"),
    case(128, 128, 256), case(128, 192, 256), case(128, 384, 256), case(256, 192, 256), case(256, 384, 1152),
    case(1, 1, 1), case(1, 8, 8, "SILU", bias="fp32"), case(2, 16, 64), case(3, 5, 7, "GELU", "fp32"), case(1, 6912, 1152, "SILU"),
    case(8, 6912, 1152), case(8, 1152, 4608, resid="fp32", gate="fp32", tokens=2), case(16, 1000, 2048, "GELU", "fp32"),
    case(17, 264, 512, resid="bf16", out=None), case(5, 100, 4096), case(32, 40, 100, out="mx"), case(1, 64, 64, out="mx"),
    case(33, 1152, 1152, "GELU"), case(64, 768, 3000, resid="bf16", gate="bf16", tokens=16), case(77, 2048, 768, bias=None),
    case(100, 40, 9000, resid="fp32"), case(129, 127, 65), case(999, 1155, 577, "SILU", resid="fp32", tokens=333),
    case(200, 333, 129, resid="bf16"), case(256, 257, 1001, "GELU", "fp32", xpad=3), case(300, 120, 136, xpad=1),
    case(31, 50, 18, xpad=1, pad=1, off=1, resid="bf16", gate="bf16"), case(257, 256, 72, resid="bf16"), case(512, 512, 512, out="fp32"),
    case(1024, 1152, 1152, "GELU", pad=8), case(1000, 4608, 1152, "GELU"), case(777, 1160, 2056, resid="fp32", out=None),
    case(2048, 3456, 1152), case(2000, 1152, 4608, resid="bf16", gate="bf16", tokens=500, inplace=True),
    case(4096, 1152, 1160, "SILU", "fp32", resid="bf16", gate="fp32", tokens=1024, bias="fp32"),
    case(130, 5000, 1536, "GELU"), case(640, 72, 16384), case(300, 136, 20000, out="fp32"), case(5000, 24, 40, resid="fp32"),
    # warps whose rows are of several samples, and columns that end inside a chunk
    case(300, 256, 320, resid="fp32", gate="bf16", tokens=1), case(300, 260, 320, resid="bf16", gate="fp32", tokens=31, pad=4),
    case(300, 264, 320, resid="fp32", gate="fp32", tokens=13, out=None), case(200, 264, 8192, resid="bf16", gate="bf16", tokens=7, out=None),
    case(5000, 264, 8192, resid="bf16", gate="bf16", tokens=33), case(2500, 1160, 5000, resid="fp32", gate="bf16", tokens=100, out="fp32"),
    # hidden states in fp32 beside outputs in fp32: the most shared memory for boxes, over short and long sums
    case(4000, 1152, 1152, resid="fp32", gate="bf16", tokens=500, out="fp32"), case(2000, 1152, 5000, resid="fp32", gate="fp32", tokens=500, out="bf16"),
    # outputs in 4 bits
    case(128, 64, 64, out="mx"), case(128, 192, 256, out="mx"), case(999, 1155, 577, "GELU", "mx"), case(256, 4608, 1152, "GELU", "mx"),
    case(1000, 1152, 4608, "SILU", "mx", xpad=2), case(300, 33, 100, out="mx"), case(400, 200, 8192, out="mx"), case(77, 31, 40, out="mx", bias="fp32"),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "{m}x{n}x{k}_{out}".format(**c))
def test_linear(lib, c):
    check(lib, c)


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(lib, seed):
    rng = np.random.default_rng(seed)
    size = lambda lo, hi: int(np.exp(rng.uniform(np.log(lo), np.log(hi))))  # noqa: E731
    pick = lambda *a: a[int(rng.integers(len(a)))]  # noqa: E731
    m, n, k = size(1, 2000), size(1, 3000), size(1, 3000)
    if rng.random() < 0.7:
        n, k = n // 8 * 8 + 8, k // 16 * 16 + 16
    resid = pick(None, "bf16", "fp32")
    c = case(m, n, k, pick("NONE", "GELU", "SILU"), pick("bf16", "fp32", "mx") if resid is None else pick("bf16", "fp32", None), resid,
             pick(None, "bf16", "fp32") if resid else None, pick("bf16", "fp32", None), int(rng.integers(0, m + 1)))
    check(lib, c, seed)


def test_every_scale_stands_at_its_own_rows_and_blocks(lib):
    """Powers of two of every size, each row's and block's another: exact sums of one term tell which was used."""
    block, cb = lib
    m, n, k = 300, 456, 640
    rng = np.random.default_rng(3)
    ex, ew = (rng.integers(107, 148, (r, k // 32)).astype(np.uint8) for r in (m, n))
    at = rng.integers(0, k, n)  # the one feature of each column that is not zero
    cx, cw = rng.integers(1, 8, (m, k)).astype(np.uint8), np.zeros((n, k), np.uint8)
    cw[np.arange(n), at] = 2  # 1.0
    x, w = (torch.from_numpy(R.packed(c)).cuda() for c in (cx, cw))
    xs, ws = torch.from_numpy(R.tiled(ex, 0xFF)).cuda(), torch.from_numpy(R.tiled(ew, 0xFF)).cuda()
    want = R.values(cx, ex, k)[:, at] * R.powers(ew)[np.arange(n), at // 32]
    for rows in (300, 128, 20):
        out = torch.zeros(rows, n, device="cuda")
        layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws)
        block.cb_linear_run(layer, block.cb_linear_io(rows=rows, out_dtype=cb.CB_FP32), x, xs, out=out)
        torch.cuda.synchronize()
        block.cb_linear_destroy(layer)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), want[:rows])


def test_the_smallest_and_largest_scales(lib):
    """Scales of 2^-127 against such of 2^127, and both in one sum: terms far apart do not disturb each other."""
    block, cb = lib
    m, n, k = 160, 72, 128
    ex, ew = np.full((m, 4), 127, np.uint8), np.full((n, 4), 127, np.uint8)
    ex[:, 0], ew[:, 0] = 0, 254
    ex[:, 1], ew[:, 1] = 254, 0
    ex[:, 2], ew[:, 2] = 0, 0  # 2^-254: nothing
    ex[5] = 0
    rng = np.random.default_rng(0)
    cx, cw = rng.integers(0, 16, (m, k)).astype(np.uint8), rng.integers(0, 16, (n, k)).astype(np.uint8)
    x, w, xs, ws = (torch.from_numpy(t).cuda() for t in (R.packed(cx), R.packed(cw), R.tiled(ex), R.tiled(ew)))
    out = torch.zeros(m, n, device="cuda")
    layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws)
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32), x, xs, out=out)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    xv, wv = R.values(cx, ex, k), R.values(cw, ew, k)
    want, size = torch.from_numpy(xv @ wv.T), torch.from_numpy(np.abs(xv) @ np.abs(wv).T)
    close(out.cpu(), want, (k + 4) * U * size + 2.0 ** -126, "fp32")


def test_blocks_that_are_not_finite_stay_apart(lib):
    block, cb = lib
    for m, n, k in ((300, 264, 192), (9, 264, 192), (130, 99, 101)):
        rng = np.random.default_rng(m)
        v, u = rng.standard_normal((m, k)), rng.standard_normal((n, k))
        v[3, 5], u[17, 70] = np.nan, np.inf
        v[4] = 0.0
        x, xs, xv, _ = operand(v)
        w, ws, wv, _ = operand(u)
        out = torch.zeros(m, n, device="cuda")
        mx, scales = torch.zeros(m, -(-n // 32) * 16, dtype=torch.uint8, device="cuda"), torch.zeros(block.cb_mx_scale_bytes(m, n), dtype=torch.uint8, device="cuda")
        layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, ws)
        block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32), x, xs, out=out)
        block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_MXFP4, out_scale=scales.data_ptr()), x, xs, out=mx)
        torch.cuda.synchronize()
        block.cb_linear_destroy(layer)
        nan = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        nan[3], nan[:, 17] = True, True
        assert torch.equal(torch.isnan(out), nan)
        fine = ~nan
        close(torch.where(fine, out, 0.0), torch.where(fine, torch.nan_to_num(xv) @ torch.nan_to_num(wv).t(), 0.0), (k + 4) * U * (torch.nan_to_num(xv).abs() @ torch.nan_to_num(wv).abs().t()), "fp32")
        e = R.from_tiles(scales.cpu().numpy(), m, -(-n // 32))
        assert ((e == 255) == nan.cpu().numpy()[:, ::32][:, :e.shape[1]] | (np.arange(e.shape[1]) == 0)).all()
        assert bool((mx.cpu()[e[:, 0] == 255, :16] == 0).all())


@pytest.mark.parametrize("c", [case(2048, 1152, 4608, resid="bf16"), case(8, 6912, 1152), case(999, 1155, 577), case(512, 1152, 1152, "GELU", "mx")],
                         ids=lambda c: "{m}x{n}x{k}_{out}".format(**c))
def test_equal_calls_give_equal_bits(lib, c):
    first = run(lib, c)[1]
    for _ in range(6):
        assert torch.equal(first, run(lib, c)[1])
