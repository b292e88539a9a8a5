"""cb_linear_run on a GPU against plain arithmetic in 64 bits.

Bounds (u = 2^-24): the products are exact in fp32, so a sum of K of them is off by (K + 1) u sum_k |x w|
at most in any order, the bound that is used for every kernel (errors of a sum that is rounded to
nearest grow with sqrt(K): a tensor core's that is cut off may reach it). Scales, bias and activation add
3 u of what they touch; GELU and SiLU have slopes below 1.2 and their exponential is off by 2 + |t| ulp,
8 u |v| + 3 u (|t| + 4) |v| with |t| <= 90 where it counts at all (beyond, the factor is 0 or 1 to fp32)."""
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
    return t.float().double()


def half_step(v, dtype):
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -126)))
    return torch.exp2(e - (8 if dtype == "bf16" else 24))


def rows_of(rows, n, pad, off, dtype, fill=None):
    """A [rows, n] view with `pad` elements between rows, `off` elements behind a boundary."""
    buf = torch.zeros(off + rows * (n + pad) + 16, dtype=torch.float32, device="cuda").to(DT[dtype])
    v = buf[off:off + rows * (n + pad)].view(rows, n + pad)[:, :n]
    if fill is not None:
        v.copy_(fill.to(DT[dtype]))
    return v


def case(m, n, k, type="bf16", act="NONE", out="bf16", resid=None, gate=None, bias="bf16", tokens=0, pad=0, off=0, xpad=0,
         xoff=0, scales=True, inplace=False):
    return dict(m=m, n=n, k=k, type=type, act=act, out=out, resid=resid, gate=gate, bias=bias, tokens=tokens, pad=pad,
                off=off, xpad=xpad, xoff=xoff, scales=scales, inplace=inplace)


CASES = [
    case(1, 1, 1), case(1, 1, 1, "e4m3"), case(1, 8, 8, act="SILU", bias="fp32"), case(2, 16, 64), case(3, 5, 7, "e4m3", "GELU"),
    # few rows: vectors, prompts
    case(1, 6912, 1152, act="SILU"), case(8, 6912, 1152), case(8, 1152, 4608, resid="fp32", gate="fp32", tokens=2),
    case(16, 1000, 2048, "e4m3", "GELU", "fp32"), case(17, 264, 512, resid="bf16", out=None), case(5, 100, 4096, "e4m3"),
    case(33, 1152, 1152, act="GELU"), case(64, 768, 3000, resid="bf16", gate="bf16", tokens=16), case(77, 2048, 768, bias=None),
    case(100, 40, 9000, "e4m3", resid="fp32"), case(128, 128, 128), case(128, 4608, 1152, "e4m3", "GELU"),
    # odd in every direction
    case(129, 127, 65), case(999, 1155, 577, act="SILU", resid="fp32", tokens=333), case(200, 333, 129, "e4m3", resid="bf16"),
    case(256, 257, 1001, "e4m3", "GELU", "fp32", xpad=3), case(300, 120, 136, xoff=1), case(300, 120, 136, "e4m3", xoff=3, xpad=5),
    case(150, 96, 200, xpad=4), case(64, 64, 64, xoff=4), case(31, 50, 18, xpad=1, xoff=1, pad=1, off=1, resid="bf16", gate="bf16"),
    # tiles of every size, tails in every direction
    case(256, 256, 64), case(257, 256, 72, resid="bf16"), case(512, 512, 512, out="fp32"), case(384, 192, 1152, "e4m3"),
    case(1024, 1152, 1152, act="GELU", pad=8), case(1000, 4608, 1152, "e4m3", "GELU"), case(777, 1160, 2056, resid="fp32", out=None),
    case(2048, 3456, 1152), case(2000, 1152, 4608, resid="bf16", gate="bf16", tokens=500, inplace=True),
    case(4096, 1152, 1160, "e4m3", "SILU", "fp32", resid="bf16", gate="fp32", tokens=1024, bias="fp32"),
    case(3000, 2000, 1000, "e4m3", scales=False, off=4), case(8192, 144, 4608, resid="fp32", tokens=4096, gate="bf16"),
    case(130, 12288, 1536, act="GELU"), case(640, 72, 16384), case(5000, 24, 40, "e4m3", resid="fp32"),
]


def run(lib, c, seed=0, stream=None):
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3, None: cb.CB_BF16}
    g = torch.Generator(device="cuda").manual_seed(seed + c["m"] + c["n"])
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    m, n, k = c["m"], c["n"], c["k"]
    d = {"x": rows_of(m, k, c["xpad"], c["xoff"], c["type"], r(m, k) + 0.1), "w": rows_of(n, k, c["xpad"], c["xoff"], c["type"], r(n, k) / k ** 0.5)}
    if c["type"] == "e4m3":
        d["w"] = rows_of(n, k, c["xpad"], c["xoff"], c["type"], 16 * r(n, k))
        if c["scales"]:
            d["xs"], d["ws"] = torch.exp(r(m)), torch.exp(r(n)) / (16 * k ** 0.5)
    samples = -(-m // c["tokens"]) if c["tokens"] else 1
    if c["bias"]:
        d["bias"] = rows_of(1, n, 0, c["off"], c["bias"], 0.3 * r(1, n))
    if c["resid"]:
        d["resid"] = rows_of(m, n, c["pad"], c["off"], c["resid"], r(m, n))
    if c["gate"]:
        d["gate"] = rows_of(samples, n, c["pad"], c["off"], c["gate"], r(samples, n))
    want = expected(c, d)
    out = rows_of(m, n, c["pad"], c["off"], c["out"], torch.full((m, n), 7.0, device="cuda")) if c["out"] else None
    xo = (d["resid"] if c["inplace"] else rows_of(m, n, c["pad"], c["off"], c["resid"])) if c["resid"] else None
    ks = k + c["xpad"]
    layer = block.cb_linear_create(d["w"], n, k, code[c["type"]], d.get("ws"), d.get("bias"), code[c["bias"]],
                                   getattr(block, "CB_ACT_" + c["act"]), w_stride=ks)
    io = block.cb_linear_io(rows=m, tokens=c["tokens"], x_stride=ks, out_stride=n + c["pad"], resid_stride=n + c["pad"],
                            resid_out_stride=n + c["pad"], gate_stride=n + c["pad"], out_dtype=code[c["out"]],
                            resid_dtype=code[c["resid"]], gate_dtype=code[c["gate"]])
    torch.cuda.synchronize()
    block.cb_linear_run(layer, io, d["x"], d.get("xs"), d.get("resid"), d.get("gate"), out, xo, stream)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    return d, want, out, xo


def expected(c, d):
    """(v, its bound) and (hidden state, its bound before rounding)."""
    x, w = f64(d["x"]), f64(d["w"])
    if "xs" in d:
        x, w = x * f64(d["xs"])[:, None], w * f64(d["ws"])[:, None]
    v, size = x @ w.t(), x.abs() @ w.abs().t()
    if "bias" in d:
        v = v + f64(d["bias"])
        size = size + f64(d["bias"]).abs()
    e = (c["k"] + 4) * U * size
    if c["act"] != "NONE":
        t = v if c["act"] == "SILU" else 1.5957691216057308 * (v + 0.044715 * v ** 3)
        e = 1.2 * e + (8 + 3 * (t.abs().clamp_max(90) + 4)) * U * v.abs()
        v = v / (1 + torch.exp(-t))
    if not c["resid"]:
        return v, e, None, None
    r = f64(d["resid"])
    g = torch.ones((), dtype=torch.float64, device="cuda")
    if "gate" in d:
        at = torch.arange(c["m"], device="cuda") // c["tokens"] if c["tokens"] else torch.zeros(c["m"], dtype=torch.long, device="cuda")
        g = f64(d["gate"])[at]
    return v, e, r + g * v, g.abs() * e + 1.01 * U * (r.abs() + (g * v).abs())


def close(got, want, slack, dtype):
    err = (f64(got) - want).abs()
    bad = ~(err <= slack + half_step(want.abs() + slack, dtype))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist(), float(err.max()))


@pytest.mark.parametrize("c", CASES, ids=lambda c: "{m}x{n}x{k}_{type}".format(**c))
def test_linear(lib, c):
    block, cb = lib
    d, (v, e, h, eh), out, xo = run(lib, c)
    assert block.cb_linear_device_status() == 0
    if out is not None:
        close(out, v, e, c["out"])
    if xo is not None:
        close(xo, h, eh, c["resid"])
    for t in (out, xo):  # what lies between rows stays as it was
        if t is not None and c["pad"] and not c["inplace"]:
            whole = torch.as_strided(t, (c["m"], c["n"] + c["pad"]), (c["n"] + c["pad"], 1), t.storage_offset())
            assert float(whole[:, c["n"]:].abs().max()) == 0.0


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(lib, seed):
    rng = np.random.default_rng(seed)
    size = lambda lo, hi: int(np.exp(rng.uniform(np.log(lo), np.log(hi))))  # noqa: E731
    pick = lambda *a: a[int(rng.integers(len(a)))]  # noqa: E731
    m, n, k = size(1, 3000), size(1, 5000), size(1, 5000)
    if rng.random() < 0.7:
        n, k = n // 8 * 8 + 8, k // 16 * 16 + 16
    resid = pick(None, "bf16", "fp32")
    c = case(m, n, k, pick("bf16", "e4m3"), pick("NONE", "GELU", "SILU"), pick("bf16", "fp32") if resid is None else pick("bf16", "fp32", None),
             resid, pick(None, "bf16", "fp32") if resid else None, pick("bf16", "fp32", None), int(rng.integers(0, m + 1)))
    d, (v, e, h, eh), out, xo = run(lib, c, seed)
    assert lib[0].cb_linear_device_status() == 0
    if out is not None:
        close(out, v, e, c["out"])
    if xo is not None:
        close(xo, h, eh, c["resid"])


@pytest.mark.parametrize("c", [case(2048, 1152, 4608, resid="bf16"), case(8, 6912, 1152), case(100, 1152, 4608, "e4m3"),
                               case(999, 1155, 577)], ids=lambda c: "{m}x{n}x{k}".format(**c))
def test_equal_calls_give_equal_bits(lib, c):
    first = run(lib, c)[2]
    for _ in range(10):
        assert torch.equal(first, run(lib, c)[2])


def test_rows_and_features_that_are_not_finite_stay_apart(lib):
    block, cb = lib
    for m, n, k in ((300, 264, 192), (9, 264, 192), (130, 99, 101)):
        x, w = torch.ones(m, k, device="cuda").bfloat16(), torch.ones(n, k, device="cuda").bfloat16()
        x[3, 5], w[17, 2] = float("nan"), float("inf")
        out = torch.zeros(m, n, device="cuda")
        layer = block.cb_linear_create(w, n, k, cb.CB_BF16)
        block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32), x, out=out)
        torch.cuda.synchronize()
        ref = x.double() @ w.double().t()
        assert torch.equal(torch.isnan(out), torch.isnan(ref)) and torch.equal(torch.isinf(out), torch.isinf(ref))
        fine = torch.isfinite(ref)
        assert torch.equal(out[fine].double(), ref[fine])
        block.cb_linear_destroy(layer)


def test_many_calls_back_to_back_on_two_streams(lib):
    """Launches that follow each other without a wait, of every kind, with their operands read by the next one."""
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: (torch.randn(s, generator=g, device="cuda") * s[-1] ** -0.5).bfloat16()  # noqa: E731
    for m in (4, 200, 2000):
        sizes = [256, 1152, 264, 1155, 512, 256]
        ws = [r(b, a) for a, b in zip(sizes, sizes[1:])]
        x = r(m, 256) * 16
        layers = [block.cb_linear_create(w, w.shape[0], w.shape[1], cb.CB_BF16) for w in ws]
        bufs = [[torch.zeros(m, w.shape[0], device="cuda", dtype=torch.bfloat16) for w in ws] for _ in range(2)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        io = block.cb_linear_io(rows=m, out_dtype=cb.CB_BF16)
        for _ in range(5):
            for s, b in zip(streams, bufs):
                y = x
                for layer, o in zip(layers, b):
                    block.cb_linear_run(layer, io, y, out=o, stream=s)
                    y = o
        torch.cuda.synchronize()
        y = x
        for w, a, b in zip(ws, *bufs):
            assert torch.equal(a, b)
            ref = y.double() @ w.double().t()
            size = y.double().abs() @ w.double().abs().t()
            close(a, ref, (w.shape[1] + 4) * U * size, "bf16")
            y = a
        assert block.cb_linear_device_status() == 0
        for layer in layers:
            block.cb_linear_destroy(layer)


def test_in_a_graph(lib):
    block, cb = lib
    x, w = torch.randn(520, 640, device="cuda").bfloat16(), torch.randn(384, 640, device="cuda").bfloat16()
    out = torch.zeros(520, 384, device="cuda")
    layer = block.cb_linear_create(w, 384, 640, cb.CB_BF16)
    io = block.cb_linear_io(rows=520, out_dtype=cb.CB_FP32)
    block.cb_linear_run(layer, io, x, out=out)
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        block.cb_linear_run(layer, io, x, out=out, stream=torch.cuda.current_stream())
    x.mul_(2)
    want = 2 * out
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    block.cb_linear_destroy(layer)


def test_row_offsets_beyond_2_31(lib):
    """Rows of the operands and of the results that begin behind 2^32 bytes."""
    block, cb = lib
    m, n, k = 40, 64, 128
    stride = 1 << 26  # elements: 40 rows span 5 GB
    x = torch.zeros(m * stride, dtype=torch.bfloat16, device="cuda").view(m, stride)
    xv = x[:, :k]
    xv.copy_(torch.randn(m, k, device="cuda"))
    out = torch.zeros(m * stride, dtype=torch.bfloat16, device="cuda").view(m, stride)
    w = torch.randn(n, k, device="cuda").bfloat16()
    layer = block.cb_linear_create(w, n, k, cb.CB_BF16)
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, x_stride=stride, out_stride=stride, out_dtype=cb.CB_BF16), x, out=out)
    torch.cuda.synchronize()
    ref = xv.double() @ w.double().t()
    close(out[:, :n], ref, (k + 4) * U * (xv.double().abs() @ w.double().abs().t()), "bf16")
    assert float(out[:, n:n + 64].abs().max()) == 0.0
    block.cb_linear_destroy(layer)


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("k", [512, 520, 4096, 16384])
def test_fp32_sums_do_not_lose_with_their_length(lib, type, k):
    """fp32 results of long sums. A part of 512 products takes 32 additions on the tensor cores, each of which cuts off half of
    2^-23 of the running sum on average, and the running sum averages two thirds of the part's: 1.3e-6 of it in all, however
    many parts are then added rounded to nearest."""
    block, cb = lib
    m, n = 384, 200
    g = torch.Generator(device="cuda").manual_seed(k)
    for shift in (0.0, 1.0):
        x = (torch.randn(m, k, generator=g, device="cuda") + shift).to(DT[type])
        w = torch.randn(n, k, generator=g, device="cuda").to(DT[type])
        r = torch.zeros(m, n, device="cuda")
        out, xo = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        layer = block.cb_linear_create(w, n, k, cb.CB_BF16 if type == "bf16" else cb.CB_E4M3)
        io = block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32, resid_dtype=cb.CB_FP32)
        block.cb_linear_run(layer, io, x, resid=r, out=out, resid_out=xo)
        torch.cuda.synchronize()
        ref = f64(x) @ f64(w).t()
        assert float((out.double() - ref).norm() / ref.norm()) < 1.3e-6
        assert torch.equal(out, xo)
        block.cb_linear_destroy(layer)


OFF_GRID = [case(40, 96, 33), case(40, 96, 31, "e4m3"), case(65, 130, 1, "e4m3"), case(300, 200, 17, "e4m3", xoff=9, xpad=2),
            case(700, 520, 1031, resid="fp32", gate="bf16", tokens=100), case(700, 520, 2063, "e4m3", out="fp32"), case(90, 700, 5494),
            case(1500, 1100, 2049, act="GELU"), case(333, 64, 4097, "e4m3", xpad=1, resid="bf16"), case(2000, 1000, 40, xoff=1)]


@pytest.mark.parametrize("c", OFF_GRID, ids=lambda c: "{m}x{n}x{k}_{type}".format(**c))
def test_operands_off_the_grid(lib, c):
    d, want, out, xo = run(lib, c, seed=5)
    v, e, hidden, he = want
    if c["out"]:
        close(out, v, e, c["out"])
    if c["resid"]:
        close(xo, hidden, he, c["resid"])


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("xoff,woff", [(0, 1), (3, 0), (5, 2)])
def test_only_the_operands_rows_are_summed(lib, type, xoff, woff):
    """One operand off the grid or both, with NaN before, between and behind the rows: none of it reaches a result."""
    block, cb = lib
    m, n, k = 200, 136, 144
    g = torch.Generator(device="cuda").manual_seed(3)
    data = {}
    for name, rows, off in (("x", m, xoff), ("w", n, woff)):
        buf = torch.full((off + rows * (k + 16) + 16,), float("nan"), device="cuda").to(DT[type])
        data[name] = buf[off:off + rows * (k + 16)].view(rows, k + 16)[:, :k]
        data[name].copy_(torch.randint(-4, 5, (rows, k), generator=g, device="cuda").to(DT[type]))
    out = torch.empty(m, n, device="cuda")
    layer = block.cb_linear_create(data["w"], n, k, cb.CB_E4M3 if type == "e4m3" else cb.CB_BF16, w_stride=k + 16)
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, x_stride=k + 16, out_dtype=cb.CB_FP32), data["x"], out=out)
    assert torch.equal(out.double(), f64(data["x"]) @ f64(data["w"]).t())  # small whole numbers: exact
    block.cb_linear_destroy(layer)


def test_off_the_grid_on_two_streams_and_in_a_graph(lib):
    """The copies of such operands: calls of several sizes on two streams at once, then some in one graph, whose inputs change."""
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(9)
    whole = lambda *s: torch.randint(-4, 5, s, generator=g, device="cuda").bfloat16()  # noqa: E731
    sets = []
    for m, n, k in [(100, 77, 333), (1000, 500, 1031), (64, 2000, 65), (513, 129, 4097)]:
        x, w = whole(m, k), whole(n, k)
        sets.append((x, w, block.cb_linear_create(w, n, k, cb.CB_BF16), block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32)))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for turn in range(40):
        for i, (x, w, layer, io) in enumerate(sets):
            out = torch.empty(x.shape[0], w.shape[0], device="cuda")
            outs.append((i, out))
    torch.cuda.synchronize()
    for j, (i, out) in enumerate(outs):
        x, w, layer, io = sets[i]
        block.cb_linear_run(layer, io, x, out=out, stream=streams[j % 2 ^ (j // 4) % 2])
    torch.cuda.synchronize()
    for i, out in outs:
        assert torch.equal(out.double(), f64(sets[i][0]) @ f64(sets[i][1]).t())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]), torch.cuda.graph(graph, stream=streams[0]):
        for i, (x, w, layer, io) in enumerate(sets):
            block.cb_linear_run(layer, io, x, out=outs[i][1], stream=torch.cuda.current_stream())
    for turn in range(3):
        for x, w, layer, io in sets:
            x.copy_(whole(*x.shape))
            w.copy_(whole(*w.shape))
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, w, layer, io) in enumerate(sets):
            assert torch.equal(outs[i][1].double(), f64(x) @ f64(w).t()), (turn, i)
    for x, w, layer, io in sets:
        block.cb_linear_destroy(layer)
    assert block.cb_linear_device_status() == 0


# few tiles of long sums: parts of K that are summed by themselves
PARTS = [case(40, 64, 16384, "e4m3", "GELU", "fp32"), case(256, 1152, 4608, resid="bf16", gate="bf16", tokens=100, inplace=True),
         case(77, 1150, 4096, out="fp32", resid="fp32", tokens=7, gate="fp32", pad=1, off=1), case(100, 33, 5001, act="SILU"),
         case(1500, 300, 12000, resid="bf16", out=None), case(64, 31, 8192, "e4m3", resid="bf16", gate="fp32", tokens=64),
         case(300, 40, 1100, bias=None), case(130, 257, 9000, out="fp32", bias="fp32", pad=3)]


@pytest.mark.parametrize("c", PARTS, ids=lambda c: "{m}x{n}x{k}_{type}".format(**c))
def test_few_tiles_of_long_sums(lib, c):
    block, cb = lib
    d, (v, e, h, eh), out, xo = run(lib, c, seed=11)
    assert block.cb_linear_device_status() == 0
    if out is not None:
        close(out, v, e, c["out"])
    if xo is not None:
        close(xo, h, eh, c["resid"])
    again = run(lib, c, seed=11)
    for a, b in ((out, again[2]), (xo, again[3])):
        assert a is None or torch.equal(a, b)
    for t in (out, xo):  # what lies between rows stays as it was
        if t is not None and c["pad"]:
            whole = torch.as_strided(t, (c["m"], c["n"] + c["pad"]), (c["n"] + c["pad"], 1), t.storage_offset())
            assert float(whole[:, c["n"]:].abs().max()) == 0.0


FIRST_IN_A_GRAPH = """
import torch
from paper_2608_23429_gb300 import block, chebboost as cb
x, w = torch.ones(100, 333, device="cuda").bfloat16(), torch.ones(50, 333, device="cuda").bfloat16()
out = torch.zeros(100, 50, device="cuda")
layer = block.cb_linear_create(w, 50, 333, cb.CB_BF16)
io = block.cb_linear_io(rows=100, out_dtype=cb.CB_FP32)
s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
    block.cb_linear_run(layer, io, x, out=out, stream=torch.cuda.current_stream())
graph.replay()
torch.cuda.synchronize()
assert bool((out == 333).all())
"""


def test_the_first_call_of_a_process_may_be_captured(lib):
    import subprocess
    import sys
    from pathlib import Path
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_GRAPH], cwd=Path(__file__).parents[1], capture_output=True, text=True, timeout=200)
    assert r.returncode == 0, r.stderr
