"""cb_linear_run whose results' rows start on 16-byte boundaries and end inside one, in bf16 and e4m3: whole pieces of 16 bytes leave by TMA, what is
behind them by the threads, and nothing else is written. Whole numbers, exact in every type."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def check(lib, type, m, n, k, wide, out, resid, gate=False, inplace=False, tokens=0):
    """Rows in a buffer that ends with the last row's last element, with a guard behind; `wide`: elements from row to row."""
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, None: cb.CB_BF16}
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda").float()  # noqa: E731
    x, w = ints(-1, 2, m, k), ints(-1, 2, n, k)
    w[:, 24:-8] = 0.0  # sums of up to 32: exact in bf16, with the hidden state too
    t = torch.bfloat16 if type == "bf16" else torch.float8_e4m3fn
    want = x @ w.t()

    def buffer(dtype, fill):
        b = torch.full(((m - 1) * wide + n + 64,), fill, device="cuda").to(DT[dtype])
        return b, b[:(m - 1) * wide + n].as_strided((m, n), (wide, 1))

    yb, y = buffer(out, 5.0) if out else (None, None)
    rb, r = buffer(resid, 6.0) if resid else (None, None)
    ob, o = (rb, r) if inplace else buffer(resid, 7.0) if resid else (None, None)
    h = None
    if resid:
        r.copy_(ints(-60, 61, m, n))
        gates = ints(0, 3, -(-m // tokens) if tokens else 1, wide) if gate else None
        h = r.float() + (want * gates[torch.arange(m, device="cuda") // (tokens or m)][:, :n] if gate else want)
    w8, x8 = w.to(t), x.to(t)
    layer = block.cb_linear_create(w8, n, k, cb.CB_BF16 if type == "bf16" else cb.CB_E4M3)
    io = block.cb_linear_io(rows=m, tokens=tokens, out_stride=wide, resid_stride=wide, resid_out_stride=wide, gate_stride=wide, out_dtype=code[out],
                            resid_dtype=code[resid], gate_dtype=cb.CB_FP32)
    block.cb_linear_run(layer, io, x8, None, rb, gates if gate else None, yb, ob)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    assert block.cb_linear_device_status() == 0
    for b, v, ref, fill in ((yb, y, want, 5.0), (ob, o, h, 6.0 if inplace else 7.0)):
        if b is None:
            continue
        assert torch.equal(v.float(), ref), (v.float() != ref).nonzero()[:3].tolist()
        assert bool((b[(m - 1) * wide + n:] == fill).all())
        assert bool((b[:(m - 1) * wide].view(m - 1, wide)[:, n:] == fill).all())


FORMS = [("bf16", None), ("fp32", None), (None, "bf16"), (None, "fp32"), ("bf16", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32")]


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("out,resid", FORMS)
def test_every_ending(lib, type, out, resid):
    """Each number of elements behind the last whole piece, and of whole pieces in the last chunk of 32 columns; fewer than a piece."""
    for n in (257, 258, 259, 260, 261, 262, 263, 265, 275, 279, 287, 33, 9, 7, 3, 1):
        check(lib, type, 45, n, 64, 288, out, resid)


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("out,resid", FORMS)
@pytest.mark.parametrize("m,n,k,wide", [(4000, 1155, 512, 1160), (3000, 2100, 1536, 2104), (900, 1154, 8192, 1184)])
def test_many_tiles(lib, type, out, resid, m, n, k, wide):
    """Several tiles a CTA, pairs of CTAs, passes over K and parts of it."""
    check(lib, type, m, n, k, wide, out, resid)
    if resid:
        check(lib, type, m, n, k, wide, out, resid, inplace=True)


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("out", ["bf16", "fp32", None])
def test_gates_that_end_on_the_grid(lib, type, out):
    """bf16 results that end inside a piece under fp32 gates that do not; rows of several samples in a warp."""
    for m, n, k, tokens in ((3000, 1156, 512, 1500), (300, 260, 64, 7), (2000, 1156, 4608, 100)):
        check(lib, type, m, n, k, n + 4, out, "bf16", gate=True, tokens=tokens)


def test_in_a_graph_and_on_two_streams(lib):
    """Calls of two streams into columns of one wider tensor, next to each other, captured and replayed: neither touches the other's."""
    block, cb = lib
    m, n, k = 1000, 300, 256
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = (torch.randint(-1, 2, (r, k), generator=g, device="cuda").bfloat16() for r in (m, 2 * n))
    both = torch.zeros(m, 608, dtype=torch.bfloat16, device="cuda")  # columns 0 to 299 and 304 to 603
    layers = [block.cb_linear_create(w[i * n:(i + 1) * n], n, k, cb.CB_BF16) for i in range(2)]
    io = block.cb_linear_io(rows=m, out_stride=608, out_dtype=cb.CB_BF16)
    want = (x.float() @ w.float().t()).bfloat16()
    streams, graphs = [torch.cuda.Stream(), torch.cuda.Stream()], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    for i, (s, graph) in enumerate(zip(streams, graphs)):
        with torch.cuda.graph(graph, stream=s):
            block.cb_linear_run(layers[i], io, x, out=both[:, 304 * i:], stream=s)
    for _ in range(5):
        both.fill_(9.0)
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(both[:, :n], want[:, :n]) and torch.equal(both[:, 304:304 + n], want[:, n:])
        assert bool((both[:, n:304] == 9.0).all()) and bool((both[:, 304 + n:] == 9.0).all())
    assert block.cb_linear_device_status() == 0
    for layer in layers:
        block.cb_linear_destroy(layer)
