"""cb_mx_quantize and cb_mx_dequantize against the format in plain numpy: equal bits, as the scales are powers of two and every
rounding is one of an exact value."""
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


def rows_of(v, dtype, pad, off):
    """v as a view with `pad` elements between rows, `off` elements behind a boundary."""
    r, k = v.shape
    buf = torch.full((off + r * (k + pad),), 77.0, dtype=DT[dtype], device="cuda")
    x = buf[off:].view(r, k + pad)[:, :k]
    x.copy_(v)
    return x


def values(r, k, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(r, k, generator=g, device="cuda") * torch.exp(2 * torch.randn(r, 1, generator=g, device="cuda"))
    return v.to(DT[dtype])


def check(lib, v, dtype, pad=0, off=0, codes_pad=0):
    block, cb = lib
    r, k = v.shape
    blocks = -(-k // 32)
    wide = 16 * blocks + codes_pad // 2
    code = cb.CB_BF16 if dtype == "bf16" else cb.CB_FP32
    x = rows_of(v, dtype, pad, off)
    codes = torch.full((r, wide), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((block.cb_mx_scale_bytes(r, k),), 0xA5, dtype=torch.uint8, device="cuda")
    d = block.cb_mx_desc(rows=r, features=k, stride=k + pad, codes_stride=2 * wide, dtype=code)
    block.cb_mx_quantize(d, x, codes, scales)
    back = rows_of(torch.full_like(v, 5.0), dtype, pad, off)
    block.cb_mx_dequantize(d, codes, scales, back)
    want = v.double().cpu().numpy()
    held, want_codes, _ = R.quantised(want)
    e = R.scale_bytes(want)
    got_codes, got_scales = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(got_scales, R.tiled(e, 0xA5))  # and nothing of the rows behind the last
    assert np.array_equal(got_codes[:, :16 * blocks], want_codes)
    assert (got_codes[:, 16 * blocks:] == 0xA5).all()
    with np.errstate(over="ignore"):
        held = torch.from_numpy(held).to(torch.float32).to(DT[dtype])
    got = back.cpu()
    assert torch.equal(torch.nan_to_num(got, nan=12345.0), torch.nan_to_num(held, nan=12345.0))
    if pad:
        between = back.as_strided((r - 1, pad), (k + pad, 1), back.storage_offset() + k)
        assert bool((between == 77.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("r,k", [(1, 1), (1, 31), (3, 32), (31, 33), (32, 64), (33, 127), (127, 128), (128, 129), (129, 255),
                                 (300, 256), (257, 257), (999, 577), (64, 1152), (5, 16384), (1000, 40)])
def test_rows(lib, r, k, dtype):
    check(lib, values(r, k, dtype, r + k), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("k,pad,off,codes_pad", [(256, 8, 0, 32), (256, 1, 0, 0), (256, 0, 1, 64), (250, 6, 8, 0), (100, 3, 5, 32),
                                                 (1152, 1152, 1152, 0), (97, 31, 4, 0)])
def test_strides_and_places(lib, k, pad, off, codes_pad, dtype):
    check(lib, values(150, k, dtype, k + pad), dtype, pad, off, codes_pad)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_special_values(lib, dtype):
    v = values(140, 160, dtype, 5)
    v[0] = 0.0
    v[1, :32] = -0.0
    v[2, 40], v[3, 41], v[4, 159] = float("nan"), float("inf"), float("-inf")
    v[5] = torch.finfo(DT[dtype]).max
    v[6] = torch.finfo(DT[dtype]).tiny
    v[7] = 2.0 ** -133
    v[8] = v[8] * 2.0 ** -125
    for i, top in enumerate((3.5, 3.484375, 6.0, 7.0, 6.96875, 1.75, 0.875 * 2.0 ** -126, 7.0 * 2.0 ** -128)):
        v[9 + i] = torch.linspace(-1, 1, 160, device="cuda") * top  # maxima on and next to the border, and of subnormal scales
        v[9 + i, ::32] = top
    grid = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5], device="cuda").repeat(2)
    for i, p in enumerate((1.0, 2.0 ** -20, 2.0 ** 60)):  # every tie
        v[20 + i] = torch.cat([grid, -grid, grid.flip(0), grid, -grid]) * p
    check(lib, v, dtype)


def test_every_code_and_scale_byte_is_read(lib):
    block, cb = lib
    r, k = 256, 64
    e = np.stack([np.arange(256), np.arange(256)[::-1]], 1).astype(np.uint8)
    c = np.tile(np.arange(16, dtype=np.uint8), (256, 4))
    codes, scales = torch.from_numpy(R.packed(c)).cuda(), torch.from_numpy(R.tiled(e)).cuda()
    for code, t in ((cb.CB_FP32, torch.float32), (cb.CB_BF16, torch.bfloat16)):
        x = torch.empty(r, k, dtype=t, device="cuda")
        block.cb_mx_dequantize(block.cb_mx_desc(rows=r, features=k, dtype=code), codes, scales, x)
        with np.errstate(over="ignore"):
            want = torch.from_numpy(R.values(c, e, k).astype(np.float32)).to(t)
        assert torch.equal(torch.nan_to_num(x.cpu(), nan=12345.0, posinf=9e37), torch.nan_to_num(want, nan=12345.0, posinf=9e37))


def test_offsets_beyond_2_31(lib):
    """Rows 2^31 + 64 elements apart."""
    block, cb = lib
    k, stride = 96, (1 << 31) + 64
    buf = torch.empty(2 * stride + k, dtype=torch.bfloat16, device="cuda")
    v = values(3, k, "bf16", 1)
    for i in range(3):
        buf[i * stride:i * stride + k] = v[i]
    codes = torch.empty(3, 48, dtype=torch.uint8, device="cuda")
    scales = torch.empty(block.cb_mx_scale_bytes(3, k), dtype=torch.uint8, device="cuda")
    d = block.cb_mx_desc(rows=3, features=k, stride=stride, dtype=cb.CB_BF16)
    block.cb_mx_quantize(d, buf, codes, scales)
    held, want, _ = R.quantised(v.double().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), want)
    block.cb_mx_dequantize(d, codes, scales, buf)
    got = torch.stack([buf[i * stride:i * stride + k] for i in range(3)])
    assert torch.equal(got.double().cpu(), torch.from_numpy(held))


def test_streams_and_graphs(lib):
    """Another stream than the current one, and a captured pair of calls replayed on new values."""
    block, cb = lib
    r, k = 200, 320
    x, back = values(r, k, "bf16", 1), torch.empty(r, k, dtype=torch.bfloat16, device="cuda")
    codes = torch.empty(r, 160, dtype=torch.uint8, device="cuda")
    scales = torch.empty(block.cb_mx_scale_bytes(r, k), dtype=torch.uint8, device="cuda")
    d = block.cb_mx_desc(rows=r, features=k, dtype=cb.CB_BF16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def calls():
        block.cb_mx_quantize(d, x, codes, scales, s)
        block.cb_mx_dequantize(d, codes, scales, back, s)

    calls()
    s.synchronize()
    assert torch.equal(back.double().cpu(), torch.from_numpy(R.quantised(x.double().cpu().numpy())[0]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        calls()
    for seed in (2, 3):
        x.copy_(values(r, k, "bf16", seed))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(back.double().cpu(), torch.from_numpy(R.quantised(x.double().cpu().numpy())[0]))
