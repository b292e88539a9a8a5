"""cb_norm_residual on a GPU against plain arithmetic in 64 bits.

Bounds (u = 2^-24), from the operations alone. h is rounded once (u |h|). The sum of squares adds
positive terms, at most hidden/32 of them by one thread, then a tree: with the roundings of h and of the
products it is off by (hidden/32 + 24) u of itself, the reciprocal root by half of that and 3 u more.
y = n (1 + s) + d adds 3 u of everything it sums. An e4m3 value is off by half its step besides."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def f64(t):
    return t.double().cpu().numpy()


def half_step(v, dtype):
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126)))
    return np.exp2(e - (8 if dtype == "bf16" else 24))


def rows_of(rows, hidden, stride, off, dtype, fill=None):
    """A [rows, hidden] view with that stride, `off` elements behind a boundary."""
    buf = torch.zeros(off + rows * stride + 16, dtype=torch.float32, device="cuda").to(DT[dtype])
    v = buf[off:off + rows * stride].view(rows, stride)[:, :hidden]
    if fill is not None:
        v.copy_(fill)
    return v


CASES = [
    # rows, hidden, tokens, x, branch, params, out, gate, weight, mod, row padding, offset
    (1, 1, 0, "fp32", "fp32", "fp32", "e4m3", True, True, True, 0, 0),
    (3, 7, 2, "bf16", "bf16", "bf16", "bf16", True, True, True, 0, 1),
    (5, 8, 1, "bf16", "bf16", "bf16", "e4m3", False, True, False, 0, 0),
    (77, 768, 0, "bf16", "bf16", "bf16", "e4m3", False, True, False, 0, 0),
    (64, 64, 16, "fp32", "bf16", "fp32", "fp32", True, False, True, 8, 0),
    (33, 264, 11, "bf16", "fp32", "fp32", "bf16", True, True, True, 0, 0),
    (999, 577, 333, "bf16", "bf16", "bf16", "bf16", True, False, True, 0, 1),
    (21, 1001, 7, "fp32", None, "bf16", "e4m3", False, True, True, 3, 1),
    (512, 1152, 256, "bf16", "bf16", "bf16", "e4m3", True, False, True, 0, 0),
    (130, 1152, 65, "fp32", "bf16", "bf16", "e4m3", True, False, True, 128, 0),
    (40, 1280, 40, "bf16", None, "bf16", "bf16", False, True, False, 0, 0),
    (40, 1288, 10, "bf16", "bf16", "bf16", "e4m3", True, True, True, 0, 0),
    (17, 2048, 4, "fp32", "fp32", "fp32", "e4m3", True, True, True, 0, 0),
    (18, 2560, 9, "bf16", "bf16", "fp32", "fp32", True, False, True, 0, 0),
    (30, 4096, 15, "bf16", "bf16", "bf16", "e4m3", True, True, True, 0, 0),
    (12, 4097, 6, "bf16", "bf16", "bf16", "e4m3", True, True, True, 0, 0),
    (9, 8192, 3, "fp32", "bf16", "bf16", "e4m3", True, False, True, 0, 0),
    (6, 16384, 2, "bf16", "bf16", "bf16", "bf16", True, True, True, 0, 0),
    (4, 9999, 2, "fp32", "fp32", "bf16", "e4m3", True, True, True, 0, 3),
    (3, 20008, 1, "bf16", "bf16", "bf16", "e4m3", True, True, True, 0, 0),
    (2, 33333, 1, "fp32", None, "fp32", "fp32", False, True, False, 1, 1),
]


def inputs(c, seed=0):
    rows, hidden, tokens, x, branch, par, out, gate, weight, mod, pad, off = c
    g = torch.Generator().manual_seed(seed + hidden)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    samples = -(-rows // tokens) if tokens else 1
    ch = torch.exp(0.7 * r(hidden))
    d = {"x": rows_of(rows, hidden, hidden + pad, off, x, r(rows, hidden) * ch)}
    if branch:
        d["branch"] = rows_of(rows, hidden, hidden + pad, off, branch, 0.5 * r(rows, hidden))
    if gate:
        d["gate"] = rows_of(samples, hidden, hidden + pad, off, par, 0.5 * r(samples, hidden))
    if weight:
        d["weight"] = rows_of(1, hidden, hidden, off, par, 1 + 0.2 * r(1, hidden))
    if mod:
        d["scale"] = rows_of(samples, hidden, hidden + pad, off, par, 0.3 * r(samples, hidden))
        d["shift"] = rows_of(samples, hidden, hidden + pad, off, par, 0.3 * r(samples, hidden))
    return d


def call(lib, c, d, x_out="new", eps=1e-6, stream=None):
    block, cb = lib
    rows, hidden, tokens, x, branch, par, out, gate, weight, mod, pad, off = c
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3, None: cb.CB_BF16}
    y = rows_of(rows, hidden, hidden + pad, off, out)
    s = torch.zeros(rows, device="cuda") if out == "e4m3" else None
    xo = rows_of(rows, hidden, hidden + pad, off, x) if x_out == "new" else d["x"] if x_out == "same" else None
    n = hidden + pad
    desc = block.cb_norm_desc(rows=rows, hidden=hidden, tokens=tokens, x_stride=n, branch_stride=n, x_out_stride=n,
                              out_stride=n, line_stride=n, x_dtype=code[x], branch_dtype=code[branch],
                              param_dtype=code[par], out_dtype=code[out], eps=eps)
    block.cb_norm_residual(desc, d["x"], d.get("branch"), d.get("gate"), d.get("weight"), d.get("scale"), d.get("shift"),
                           xo, y, s, stream)
    return xo, y, s


def expected(c, d, eps=1e-6):
    rows, hidden, tokens = c[:3]
    at = np.arange(rows) // tokens if tokens else np.zeros(rows, dtype=int)
    h = f64(d["x"])
    size = np.abs(h)
    if "branch" in d:
        b = f64(d["branch"]) * (f64(d["gate"])[at] if "gate" in d else 1.0)
        h, size = h + b, size + np.abs(b)
    n = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    if "weight" in d:
        n = n * f64(d["weight"])
    s = f64(d["scale"])[at] if "scale" in d else 0.0
    t = f64(d["shift"])[at] if "shift" in d else 0.0
    y = n * (1 + s) + t
    rel = ((hidden / 32 + 24) / 2 + 5) * U
    return h, U * np.abs(h), y, rel * np.abs(n) * (1 + np.abs(s)) + 3 * U * (np.abs(n) * (1 + np.abs(s)) + np.abs(t))


def check(c, d, got, want):
    xo, y, s = got
    h, eh, ref, ey = want
    if xo is not None:
        assert (np.abs(f64(xo) - h) <= eh + half_step(np.abs(h) + eh, c[3])).all()
    if c[6] != "e4m3":
        err = np.abs(f64(y) - ref)
        assert (err <= ey + half_step(np.abs(ref) + ey, c[6])).all(), float((err - ey).max())
        return
    s = f64(s)[:, None]
    top = np.abs(ref).max(1, keepdims=True)
    assert (np.abs(s - np.maximum(top / 448, 2.0 ** -126)) <= (ey.max(1, keepdims=True) + 3 * U * top) / 448).all()
    v = np.abs(ref / s) * (1 + 4 * U) + ey / s
    step = np.where(v >= 2.0 ** -6, np.exp2(np.floor(np.log2(np.maximum(v, 2.0 ** -20))) - 3), 2.0 ** -9)
    err = np.abs(f64(y.float()) * s - ref)
    assert (err <= ey + s * (0.5 * step + 4 * U * v)).all(), float((err / s).max())


@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c[:2])))
@pytest.mark.parametrize("x_out", ["new", "same", None])
def test_norm(lib, c, x_out):
    d = inputs(c)
    want = expected(c, d)
    got = call(lib, c, d, x_out)
    torch.cuda.synchronize()
    check(c, d, got, want)


def test_padding_between_rows_is_not_written(lib):
    c = (9, 72, 3, "bf16", "bf16", "bf16", "e4m3", True, True, True, 8, 0)
    d = inputs(c)
    xo, y, s = call(lib, c, d)
    torch.cuda.synchronize()
    for v in (xo, y):
        whole = torch.as_strided(v, (9, 80), (80, 1)).float()
        assert float(whole[:, 72:].abs().max()) == 0.0 and float(whole[:, :72].abs().max()) > 0


@pytest.mark.parametrize("hidden", [40, 1152, 4104, 1153, 20001])
def test_rows_of_zeros_and_of_values_that_are_not_finite(lib, hidden):
    c = (6, hidden, 0, "fp32", "fp32", "fp32", "e4m3", False, True, False, 0, 0)
    d = inputs(c)
    d["x"][1].zero_(), d["branch"][1].zero_()
    d["x"][3, hidden // 2] = float("nan")
    d["branch"][4, hidden - 1] = float("inf")
    d["x"][5] *= 1e-30
    d["branch"][5] *= 1e-30
    xo, y, s = call(lib, c, d)
    torch.cuda.synchronize()
    v = y.float()
    assert float(v[1].abs().max()) == 0.0 and float(s[1]) == 2.0 ** -126
    assert bool(torch.isnan(v[3]).all()) and bool(torch.isnan(v[4]).all())
    for r in (0, 2, 5):
        assert bool(torch.isfinite(v[r]).all()) and float(v[r].abs().max()) == 448.0 and math.isfinite(float(s[r]))


def test_side_stream_and_no_rows(lib):
    block, cb = lib
    c = CASES[8]
    d = inputs(c)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = call(lib, c, d, stream=st)
    st.synchronize()
    check(c, d, got, expected(c, d))
    desc = block.cb_norm_desc(rows=0, hidden=8, x_dtype=cb.CB_BF16, out_dtype=cb.CB_BF16, eps=0.0)
    block.cb_norm_residual(desc, None, out=None)
    # nothing but x: a plain norm of 16-bit rows
    x = torch.randn(5, 96, device="cuda").bfloat16()
    out = torch.zeros(5, 96, device="cuda")
    desc = block.cb_norm_desc(rows=5, hidden=96, x_dtype=cb.CB_BF16, out_dtype=cb.CB_FP32, eps=1e-5)
    block.cb_norm_residual(desc, x, out=out)
    ref = f64(x) / np.sqrt((f64(x) ** 2).mean(1, keepdims=True) + 1e-5)
    assert (np.abs(f64(out) - ref) <= 30 * U * np.abs(ref)).all()


@pytest.mark.parametrize("hidden", [40, 1152, 1153, 3080])
def test_an_infinite_gate_spoils_its_own_column_only(lib, hidden):
    """The row's sum is infinite: the column itself is NaN, all others are what zeros give."""
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(hidden)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, branch, gate, scale, shift = r(6, hidden), r(6, hidden) + 4, r(2, hidden), r(2, hidden), r(2, hidden)
    gate[1, 3] = float("inf")
    out = torch.empty(6, hidden, device="cuda")
    desc = block.cb_norm_desc(rows=6, hidden=hidden, tokens=3, out_dtype=cb.CB_FP32, eps=1e-6)
    block.cb_norm_residual(desc, x, branch, gate, None, scale, shift, None, out)
    want = shift[1].float().expand(3, hidden)
    assert torch.isfinite(out[:3]).all() and torch.isnan(out[3:, 3]).all()
    others = torch.arange(hidden, device="cuda") != 3
    assert torch.equal(out[3:, others], want[:, others])


@pytest.mark.parametrize("hidden", [8, 9, 15, 63, 250, 577, 1151, 1267, 2041, 3001, 4097, 8187, 16370, 16383])
@pytest.mark.parametrize("x,branch,out", [("bf16", "bf16", "e4m3"), ("fp32", "bf16", "bf16"), ("bf16", "fp32", "fp32"), ("fp32", None, "e4m3")])
def test_rows_off_the_grid(lib, hidden, x, branch, out):
    """Contiguous rows whose starts take every place of a vector, lines in bf16 off the grid as well, in place."""
    c = (45, hidden, 9, x, branch, "bf16", out, branch is not None, True, True, 0, 0)
    d = inputs(c, seed=2)
    want = expected(c, d)
    check(c, d, call(lib, c, d, "same"), want)


@pytest.mark.parametrize("hidden", [250, 1151])
def test_only_the_row_s_own_elements_count(lib, hidden):
    """Rows of NaN among others, and gates of NaN for the other samples."""
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(hidden)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, branch, gate, scale = r(9, hidden), r(9, hidden), r(3, hidden), r(3, hidden)
    desc = block.cb_norm_desc(rows=9, hidden=hidden, tokens=3, out_dtype=cb.CB_FP32, eps=1e-6)
    whole, out = torch.empty(9, hidden, device="cuda"), torch.empty(9, hidden, device="cuda")
    block.cb_norm_residual(desc, x, branch, gate, None, scale, None, None, whole)
    x[3], branch[5], gate[0], scale[2] = float("nan"), float("inf"), float("nan"), float("inf")
    block.cb_norm_residual(desc, x, branch, gate, None, scale, None, None, out)
    assert torch.equal(out[4], whole[4]) and torch.isnan(out[:4]).all() and torch.isnan(out[5]).any()
