"""cb_norm_around on a GPU against plain arithmetic in 64 bits.

Bounds (u = 2^-24, L = 64 + hidden / 256 additions in a row at most): a value that goes into a norm with an error e comes out of it as follows.
Mean: off by dm = mean(e) + (L + 2) u mean|v|. Difference d = v - mean: by ed = e + dm + u |d| (root mean square: e). Squares: their
mean by 2 mean(|d| ed) + mean(ed^2) + (L + 2) u mean(d^2), half of that relative for the root, and 4 u. n = d rstd: by ed rstd and that relative
to n. Each product or sum that follows adds u of its result (lines are exact)."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def half_step(v, dtype):
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -126)))
    return torch.exp2(e - (8 if dtype == "bf16" else 24))


def rows_of(v, pad, off, dtype):
    r, n = v.shape
    buf = torch.zeros(off + r * (n + pad) + 16, dtype=torch.float32, device="cuda").to(DT[dtype])
    x = buf[off:off + r * (n + pad)].view(r, n + pad)[:, :n]
    x.copy_(v.to(DT[dtype]))
    return x


def case(rows, hidden, after="none", before="layer", x="bf16", branch="bf16", param="bf16", out="bf16", gate=True, lines=True, modulated=True,
         tokens=0, factors=(1.0, 1.0), pad=0, off=0, x_out=True, mean=0.0, inplace=False, eps=1e-6):
    return dict(rows=rows, hidden=hidden, after=after, before=before, x=x, branch=branch, param=param, out=out, gate=gate, lines=lines,
                modulated=modulated, tokens=tokens, factors=factors, pad=pad, off=off, x_out=x_out, mean=mean, inplace=inplace, eps=eps)


def normed(v, e, kind, eps, L):
    """(n, its error) of values v with errors e."""
    if kind == "none":
        return v, e
    d, ed = v, e
    if kind == "layer":
        d = v - v.mean(1, keepdim=True)
        ed = e + e.mean(1, keepdim=True) + (L + 2) * U * v.abs().mean(1, keepdim=True) + U * d.abs()
    ms = (d * d).mean(1, keepdim=True)
    ems = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (L + 2) * U * ms
    rstd = 1 / torch.sqrt(ms + eps)
    rel = 0.5 * ems / (ms + eps).clamp_min(1e-300) + 4 * U
    n = d * rstd
    return n, (ed * rstd + n.abs() * rel) * (1 + rel)


def run(lib, c, seed=0, stream=None):
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3, "mx": cb.CB_MXFP4, None: cb.CB_BF16}
    kind = {"none": block.CB_NORM_NONE, "rms": block.CB_NORM_RMS, "layer": block.CB_NORM_LAYER}
    g = torch.Generator(device="cuda").manual_seed(seed + c["rows"] + c["hidden"])
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    m, n = c["rows"], c["hidden"]
    samples = -(-m // c["tokens"]) if c["tokens"] else 1
    t = {"x": rows_of(r(m, n) * torch.exp(0.5 * r(n)) + c["mean"], c["pad"], c["off"], c["x"])}
    if c["branch"]:
        t["branch"] = rows_of(0.7 * r(m, n) + c["mean"], c["pad"], c["off"], c["branch"])
        if c["gate"]:
            t["gate"] = rows_of(0.5 * r(samples, n), c["pad"], c["off"], c["param"])
    for which in ("after", "before"):
        if c["lines"] and c[which] != "none" and (which == "after" or c["out"]):
            t[which + "_weight"] = rows_of(1 + 0.3 * r(1, n), 0, c["off"], c["param"])
            t[which + "_bias"] = rows_of(0.3 * r(1, n), 0, c["off"], c["param"])
    if c["modulated"] and c["out"]:
        t["scale"], t["shift"] = (rows_of(0.4 * r(samples, n), c["pad"], c["off"], c["param"]) for _ in range(2))
    f = {k: v.double() for k, v in t.items()}
    at = torch.arange(m, device="cuda") // (c["tokens"] or m)
    L, fx, fb = 64 + n / 256, *c["factors"]
    # the formulas, and what fp32 may make of them
    h = fx * f["x"]
    eh = (0 if fx == 1 else U) * h.abs()
    if c["branch"]:
        b, eb = normed(f["branch"], torch.zeros_like(f["branch"]), c["after"], c["eps"], L)
        if "after_weight" in t:
            eb = eb * f["after_weight"].abs() + U * (b * f["after_weight"]).abs()
            b = b * f["after_weight"] + f["after_bias"]
            eb = eb + U * b.abs()
        if "gate" in t:
            eb = eb * f["gate"][at].abs() + U * (b * f["gate"][at]).abs()
            b = b * f["gate"][at]
        h, eh = h + fb * b, eh + abs(fb) * eb
        eh = 1.001 * eh + U * h.abs() + (0 if fb == 1 else U) * (fb * b).abs()
    y, ey = normed(h, eh, c["before"], c["eps"], L)
    if "before_weight" in t:
        ey = ey * f["before_weight"].abs() + U * (y * f["before_weight"]).abs()
        y = y * f["before_weight"] + f["before_bias"]
        ey = ey + U * y.abs()
    if "scale" in t:
        s = f["scale"][at]
        ey = ey * (1 + s).abs() + 2 * U * (y.abs() * (1 + s.abs()))
        y = y * (1 + s) + f["shift"][at]
        ey = ey + U * y.abs()
    ey = 1.001 * ey
    x_out = (t["x"] if c["inplace"] else rows_of(torch.full((m, n), 3.0, device="cuda"), c["pad"], c["off"], c["x"])) if c["x_out"] else None
    out = out_scale = None
    stride = n + c["pad"]
    out_stride = stride
    if c["out"] == "mx":
        out_stride = -(-n // 32) * 32 + (32 if c["pad"] else 0)
        out = torch.full((m, out_stride // 2), 0xA5, dtype=torch.uint8, device="cuda")
        out_scale = torch.full((block.cb_mx_scale_bytes(m, n),), 0xA5, dtype=torch.uint8, device="cuda")
    elif c["out"]:
        out = rows_of(torch.full((m, n), 3.0, device="cuda"), c["pad"], c["off"], c["out"])
        if c["out"] == "e4m3":
            out_scale = torch.zeros(m, device="cuda")
    d = block.cb_norm_around_desc(rows=m, hidden=n, tokens=c["tokens"], x_stride=stride, branch_stride=stride, x_out_stride=stride,
                                  out_stride=out_stride, line_stride=stride, x_dtype=code[c["x"]], branch_dtype=code[c["branch"]],
                                  param_dtype=code[c["param"]], out_dtype=code[c["out"]], after=kind[c["after"]], before=kind[c["before"]],
                                  after_eps=c["eps"], before_eps=c["eps"], x_factor=fx, branch_factor=fb)
    torch.cuda.synchronize()
    block.cb_norm_around(d, t["x"], t.get("branch"), t.get("gate"), t.get("after_weight"), t.get("after_bias"), t.get("before_weight"),
                         t.get("before_bias"), t.get("scale"), t.get("shift"), x_out, out, out_scale, stream)
    torch.cuda.synchronize()
    return (h, eh, y, ey), x_out, out, out_scale


def close(got, want, slack, dtype):
    err = (got.double() - want).abs()
    bad = ~(err <= slack + half_step(want.abs() + slack, dtype))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist(), float(err.max()))


def check(lib, c, seed=0):
    (h, eh, y, ey), x_out, out, s = run(lib, c, seed)
    if x_out is not None:
        close(x_out, h, eh, c["x"])
    if c["out"] == "mx":
        R.check_quantised(y.cpu().numpy(), ey.cpu().numpy(), out.cpu().numpy(), s.cpu().numpy())
    elif c["out"] == "e4m3":
        top, et = y.abs().amax(1), ey.amax(1)
        want = (top / 448).clamp_min(2.0 ** -126)
        assert bool(((s.double() - want).abs() <= et / 448 + 3 * U * want).all())
        step = torch.maximum(2.0 ** -4 * (y.abs() + ey), 2.0 ** -10 * s.double()[:, None])  # half of e4m3's, or of its subnormals'
        assert bool(((out.double() * s.double()[:, None] - y).abs() <= ey + 3 * U * y.abs() + step).all())
    elif c["out"]:
        close(out, y, ey, c["out"])
    for t, fill in ((x_out, 0.0), (out, 0.0)):  # what lies between rows stays as it was
        if t is not None and t.dtype != torch.uint8 and c["pad"] and not (t is x_out and c["inplace"]):
            n, p = c["hidden"], c["pad"]
            whole = torch.as_strided(t, (c["rows"], n + p), (n + p, 1), t.storage_offset())
            assert float(whole[:, n:].float().abs().max()) == fill


KINDS = [(a, b) for a in ("none", "rms", "layer") for b in ("none", "rms", "layer")]


@pytest.mark.parametrize("a,b", KINDS)
@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3", "mx"])
def test_kinds(lib, a, b, out):
    check(lib, case(70, 768, a, b, out=out, tokens=20))
    check(lib, case(70, 769, a, b, out=out, tokens=20))
    check(lib, case(33, 2056, a, b, "fp32", "fp32", "fp32", out, factors=(1.5, 0.25)))


@pytest.mark.parametrize("hidden", [1, 7, 8, 24, 33, 40, 96, 256, 264, 512, 520, 577, 768, 1152, 1280, 1288, 2048, 2056, 2500, 4096, 4104, 8192, 8200,
                                    16384, 16392, 16000, 49152, 50001])
def test_sizes(lib, hidden):
    rows = 150 if hidden < 3000 else 9
    for after, before, out, x in (("rms", "layer", "mx", "bf16"), ("layer", "rms", "bf16", "fp32"), ("none", "layer", "e4m3", "bf16")):
        if hidden > 1 or before != "layer":  # (one element is its own mean)
            check(lib, case(rows, hidden, after, before, x, out=out, tokens=50))


@pytest.mark.parametrize("rows,hidden", [(3, 1281), (141, 1500), (300, 2047), (310, 2047), (150, 2049), (150, 2500), (141, 3383), (160, 3383), (3, 4095), (150, 4096)])
def test_few_long_rows(lib, rows, hidden):
    """Off the 16-byte grid, as many as have an SM's warps between them at once, and a few more."""
    gap = 1 if hidden == 4096 else 0
    for after, before, out, x in (("rms", "layer", "mx", "bf16"), ("layer", "rms", "bf16", "fp32"), ("layer", "layer", "e4m3", "bf16")):
        check(lib, case(rows, hidden, after, before, x, out=out, tokens=47, pad=gap, off=gap))


@pytest.mark.parametrize("hidden", [2, 62, 66, 130, 194, 258, 382, 390, 514, 642, 770, 1026, 1282, 2050, 2562, 4098, 5122, 6146, 8190, 8194])
def test_rows_by_pairs(lib, hidden):
    """Even rows off the 16-byte grid: lengths off it, starts off it, and starts and strides that are odd, which go one by one."""
    rows = 141 if hidden < 3000 else 9
    for after, before, out, x, gap in (("rms", "layer", "mx", "bf16", 0), ("layer", "rms", "bf16", "fp32", 2), ("none", "layer", "e4m3", "bf16", 6),
                                       ("layer", "layer", "fp32", "fp32", 3)):
        if hidden > 2 or before != "layer":  # (two elements are their mean and as much off it on each side)
            check(lib, case(rows, hidden, after, before, x, out=out, tokens=50, pad=gap, off=gap))


@pytest.mark.parametrize("hidden", [254, 255, 257, 258, 382, 383, 385, 386, 511, 577, 638, 640, 641, 642, 766, 767, 768, 769, 770])
def test_many_short_rows_by_elements(lib, hidden):
    """More rows than have four warps each at once, in a number that fills no CTA."""
    pad = 1 if hidden % 8 == 0 else 0
    for after, before, out, x in (("rms", "layer", "mx", "bf16"), ("layer", "rms", "bf16", "fp32"), ("none", "layer", "e4m3", "bf16"), ("layer", "layer", "fp32", "fp32")):
        check(lib, case(2051, hidden, after, before, x, out=out, tokens=700, pad=0 if out == "mx" else pad, off=0 if out == "mx" else pad))


@pytest.mark.parametrize("c", [
    case(200, 256, pad=8, off=8), case(200, 256, pad=1, off=1), case(200, 250, pad=6, off=3), case(129, 1152, pad=1152, off=1152, out="mx"),
    case(129, 1152, pad=4, out="mx"), case(130, 130, pad=3, out="mx", x="fp32"), case(64, 640, pad=4, x="fp32", branch="fp32", param="fp32", out="fp32"),
    case(300, 384, inplace=True, tokens=7), case(300, 385, inplace=True, tokens=7), case(5, 60000, "rms", inplace=True, out="e4m3"),
    case(100, 320, x_out=False), case(100, 321, x_out=False, out="mx"), case(100, 320, "layer", "none", out=None), case(3, 60000, "layer", "none", out=None),
    case(100, 321, "rms", "none", out=None, gate=False), case(100, 320, branch=None, out="e4m3"), case(100, 321, branch=None, before="rms", out="mx"),
    case(100, 320, branch=None, x_out=False, lines=False, modulated=False), case(1, 1152), case(1, 1153), case(4099, 64, "rms", "rms", out="mx", tokens=1),
    case(2, 320, mean=100.0, x="fp32"), case(50, 1152, "layer", "layer", x="fp32", branch="fp32", mean=300.0, out="fp32"),
    case(50, 1153, "layer", "layer", x="fp32", branch="fp32", mean=300.0, out="fp32"), case(77, 768, "layer", "layer", mean=3.0, gate=False),
    case(20, 512, eps=0.0), case(20, 2048, "rms", "rms", eps=0.1)], ids=str)
def test_forms(lib, c):
    check(lib, c)


@pytest.mark.parametrize("seed", range(32))
def test_random(lib, seed):
    rng = np.random.default_rng(seed)
    pick = lambda *a: a[int(rng.integers(len(a)))]  # noqa: E731
    rows, hidden = int(np.exp(rng.uniform(0, 7))), int(np.exp(rng.uniform(np.log(2), np.log(9000))))
    if rng.random() < 0.6:
        hidden = hidden // 8 * 8 + 8
    branch = pick("bf16", "fp32", None)
    c = case(rows, hidden, pick("none", "rms", "layer") if branch else "none", pick("none", "rms", "layer"), pick("bf16", "fp32"), branch,
             pick("bf16", "fp32"), pick("bf16", "fp32", "e4m3", "mx"), rng.random() < 0.6, rng.random() < 0.6, rng.random() < 0.6,
             int(rng.integers(0, rows + 1)), pick((1.0, 1.0), (0.5, -2.0), (1.0, 0.0)), pick(0, 0, 1, 8), pick(0, 0, 1, 8), rng.random() < 0.8)
    check(lib, c, seed)


def test_rows_that_are_not_finite_stay_apart(lib):
    block, cb = lib
    for hidden in (256, 2056, 257):
        for out_dtype in (cb.CB_FP32, cb.CB_MXFP4):
            g = torch.Generator(device="cuda").manual_seed(1)
            x = torch.randn(40, hidden, generator=g, device="cuda")
            b = torch.randn(40, hidden, generator=g, device="cuda")
            outs = []
            for dirty in (False, True):
                xx, bb = x.clone(), b.clone()
                if dirty:
                    xx[3, 5], xx[9, 77], bb[20, 1], bb[21, 200] = float("nan"), float("inf"), float("-inf"), float("nan")
                xx[30] = 0.0
                bb[30] = 0.0
                o = torch.zeros(40, hidden, device="cuda") if out_dtype == cb.CB_FP32 else torch.zeros(40, -(-hidden // 32) * 16, dtype=torch.uint8, device="cuda")
                s = None if out_dtype == cb.CB_FP32 else torch.zeros(block.cb_mx_scale_bytes(40, hidden), dtype=torch.uint8, device="cuda")
                d = block.cb_norm_around_desc(rows=40, hidden=hidden, x_dtype=cb.CB_FP32, branch_dtype=cb.CB_FP32, out_dtype=out_dtype,
                                              after=block.CB_NORM_LAYER, before=block.CB_NORM_RMS, after_eps=1e-6, before_eps=1e-6)
                block.cb_norm_around(d, xx, bb, out=o, out_scale=s)
                torch.cuda.synchronize()
                outs.append((o, None if s is None else R.from_tiles(s.cpu().numpy(), 40, -(-hidden // 32))))
            (clean, cs), (got, gs) = outs
            bad = [3, 9, 20, 21]
            rest = [i for i in range(40) if i not in bad]
            assert torch.equal(clean[rest], got[rest]) and float(got[30].float().abs().max()) == 0.0
            if gs is None:
                assert bool((~torch.isfinite(got[bad])).any(1).all())
            else:
                assert np.array_equal(cs[rest], gs[rest]) and (gs[[3, 20, 21]] == 255).all() and (gs[9] == 255).any()


def test_streams_graphs_and_equal_bits(lib):
    block, cb = lib
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for c in (case(300, 1152, "rms", out="mx", tokens=100), case(300, 577, "layer", "rms", out="bf16")):
        a, b = run(lib, c), run(lib, c, stream=s)
        for p, q in zip(a[1:], b[1:]):
            assert p is None or torch.equal(p, q)
    m, n = 200, 640
    x, br = torch.randn(m, n, device="cuda").bfloat16(), torch.randn(m, n, device="cuda").bfloat16()
    xo, out = torch.empty_like(x), torch.empty_like(x)
    d = block.cb_norm_around_desc(rows=m, hidden=n, x_dtype=cb.CB_BF16, out_dtype=cb.CB_BF16, after=block.CB_NORM_RMS, before=block.CB_NORM_LAYER,
                                  after_eps=1e-6, before_eps=1e-6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        block.cb_norm_around(d, x, br, x_out=xo, out=out, stream=s)
    for _ in range(2):
        x.copy_(torch.randn(m, n, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        first = xo.clone(), out.clone()
        block.cb_norm_around(d, x, br, x_out=xo, out=out)
        torch.cuda.synchronize()
        assert torch.equal(first[0], xo) and torch.equal(first[1], out)


def test_offsets_beyond_2_31(lib):
    block, cb = lib
    n, stride = 96, (1 << 31) + 64
    buf = torch.zeros(2 * stride + n, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(3, n, device="cuda").bfloat16()
    for i in range(3):
        buf[i * stride:i * stride + n] = v[i]
    out, want = torch.empty(3, n, device="cuda"), torch.empty(3, n, device="cuda")
    kw = dict(rows=3, hidden=n, x_dtype=cb.CB_BF16, out_dtype=cb.CB_FP32, before=block.CB_NORM_LAYER, before_eps=1e-6)
    block.cb_norm_around(block.cb_norm_around_desc(x_stride=stride, x_out_stride=stride, **kw), buf, x_out=buf, out=out)
    block.cb_norm_around(block.cb_norm_around_desc(**kw), v, out=want)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(torch.stack([buf[i * stride:i * stride + n] for i in range(3)]), v)
