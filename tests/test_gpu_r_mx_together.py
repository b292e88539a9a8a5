"""The operators in 4 bits together, as they are used: the example's steps against the same blocks in 64 bits, the whole sequence in one graph, calls
on two streams, far offsets, and waits that run out.

Bounds of the example's branches (2-norm, relative): a code with one bit behind the leading one is off by at most 2^-2 of its value and evenly
so, 2^-2 / sqrt(3) = 0.144 (the weights are taken as they are); GELU's slope against its value may raise the error of its argument by half, its result
is rounded anew, and independent errors add by squares: sqrt((1.5 0.144)^2 + 0.144^2) = 0.26, which products keep; bf16 adds 2e-3. A prediction
raises it by 2.3 and adds 2.3 times the history's 6.1e-3 (test_gpu_h_mlp_branch.py)."""
import os
import sys
import time

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


@pytest.mark.parametrize("depth,batch,tokens,hidden", [(1, 2, 77, 768), (4, 2, 256, 1152), (3, 3, 50, 136)])
def test_example(lib, depth, batch, tokens, hidden):
    from paper_2608_23429_gb300 import mlp_branch
    m, off = mlp_branch.run(depth, batch, tokens, hidden, dtype=torch.float64, bits=4)
    m.close()
    branch = (1.5 ** 2 + 1) ** 0.5 * 0.144 + 2e-3
    for t, rel, change in off[:-1]:
        assert change < branch, (t, rel, change)
    assert off[-1][2] < 2.3 * (branch + 6.1e-3), off[-1]


def test_bits_are_checked(lib):
    from paper_2608_23429_gb300 import mlp_branch
    with pytest.raises(ValueError):
        mlp_branch.MlpBranches(1, 1, 1, 64, [2.0, 1.0], bits=5)


class Sequence:
    """Rows in bf16 -> norms on both sides -> 4 bits -> GELU -> 4 bits -> gated hidden state and branch; sums in parts of K on the way."""

    def __init__(self, lib, tokens, hidden, wide, batch=2):
        from paper_2608_23429_gb300 import mlp_branch as M
        self.block, self.cb = block, cb = lib
        g = torch.Generator(device="cuda").manual_seed(tokens)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        rows = self.rows = batch * tokens
        self.x, self.branch = r(rows, hidden).bfloat16(), r(rows, hidden).bfloat16()
        self.gate, self.gate2, self.scale, self.shift = (0.5 * r(4, batch, hidden)).bfloat16()
        self.weight = (1 + 0.1 * r(hidden)).bfloat16()
        self.w1, self.w2 = M.quantised(r(wide, hidden) / hidden ** 0.5), M.quantised(r(hidden, wide) / wide ** 0.5)
        self.b1, self.b2 = r(wide).bfloat16(), r(hidden).bfloat16()
        self.rows4, self.mid4, self.again4 = M.mx_buffer(rows, hidden), M.mx_buffer(rows, wide), M.mx_buffer(rows, hidden)
        self.first = block.cb_linear_create(self.w1[0], wide, hidden, cb.CB_MXFP4, self.w1[1], self.b1, activation=block.CB_ACT_GELU)
        self.second = block.cb_linear_create(self.w2[0], hidden, wide, cb.CB_MXFP4, self.w2[1], self.b2)
        self.h, self.out, self.back = (torch.empty_like(self.x) for _ in range(3))
        self.norm = block.cb_norm_around_desc(rows=rows, hidden=hidden, tokens=tokens, out_dtype=cb.CB_MXFP4, after=block.CB_NORM_RMS,
                                              before=block.CB_NORM_LAYER, after_eps=1e-6, before_eps=1e-6, branch_factor=0.5)
        self.io1 = block.cb_linear_io(rows=rows, out_dtype=cb.CB_MXFP4, out_scale=self.mid4[1].data_ptr())
        self.io2 = block.cb_linear_io(rows=rows, tokens=tokens)
        self.mx = block.cb_mx_desc(rows=rows, features=hidden)

    def run(self, s=None):
        block = self.block
        block.cb_norm_around(self.norm, self.x, self.branch, self.gate, self.weight, None, None, None, self.scale, self.shift, self.h, *self.rows4, s)
        block.cb_linear_run(self.first, self.io1, *self.rows4, out=self.mid4[0], stream=s)
        block.cb_linear_run(self.second, self.io2, *self.mid4, self.h, self.gate2, self.out, self.h, s)
        block.cb_mx_quantize(self.mx, self.h, *self.again4, s)
        block.cb_mx_dequantize(self.mx, *self.again4, self.back, s)

    def results(self):
        return [t.clone() for t in (self.h, self.out, self.back, self.rows4[0], self.mid4[0])]

    def close(self):
        self.block.cb_linear_destroy(self.first)
        self.block.cb_linear_destroy(self.second)


@pytest.mark.parametrize("tokens,hidden,wide", [(128, 1152, 4608), (333, 577, 1155), (1, 64, 96), (40, 72, 16384)])
def test_sequence_step_by_step(lib, tokens, hidden, wide):
    """Every call on what the one before left, each against 64 bits on the bytes that it was given."""
    q = Sequence(lib, tokens, hidden, wide)
    q.run()
    torch.cuda.synchronize()
    assert q.block.cb_linear_device_status() == 0
    values = lambda b, k: torch.from_numpy(R.values(R.unpacked(b[0].cpu().numpy()), R.from_tiles(b[1].cpu().numpy(), b[0].shape[0], -(-k // 32)), k)).cuda()  # noqa: E731
    x, mid, w1, w2 = values(q.rows4, hidden), values(q.mid4, wide), values(q.w1, hidden), values(q.w2, wide)
    v = x @ w1.t() + q.b1.double()
    t = 1.5957691216057308 * (v + 0.044715 * v ** 3)
    e = 1.2 * (hidden + 4) * U * (x.abs() @ w1.abs().t() + q.b1.double().abs()) + (8 + 3 * (t.abs().clamp_max(90) + 4)) * U * v.abs()
    R.check_quantised((v / (1 + torch.exp(-t))).cpu().numpy(), e.cpu().numpy(), q.mid4[0].cpu().numpy(), q.mid4[1].cpu().numpy(), 0)
    v = mid @ w2.t() + q.b2.double()
    e = (wide + 4) * U * (mid.abs() @ w2.abs().t() + q.b2.double().abs())
    assert bool(((q.out.double() - v).abs() <= e + 2.0 ** -8 * (v.abs() + e)).all())
    n = q.branch.double()
    n = 0.5 * n / torch.sqrt((n * n).mean(1, keepdim=True) + 1e-6) * q.weight.double() * q.gate.double().repeat_interleave(tokens, 0)
    h, g = q.x.double() + n, q.gate2.double().repeat_interleave(tokens, 0)
    before = h.bfloat16().double()  # held in bf16 between the calls: off by its step where h is next to a border
    want = before + g * v
    slack = g.abs() * e + 2.0 ** -8 * want.abs() + 2.0 ** -7 * h.abs() * ((h.bfloat16().double() - h).abs() > 0.98 * 2.0 ** -9 * h.abs())
    assert bool(((q.h.double() - want).abs() <= slack + 1e-6).all())
    assert np.array_equal(q.again4[0].cpu().numpy(), R.quantised(q.h.double().cpu().numpy())[1])
    q.close()


def test_sequence_in_a_graph_and_on_two_streams(lib):
    q = [Sequence(lib, 100, 640, 4608), Sequence(lib, 37, 577, 1155)]
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    sources = [[torch.randn_like(a.x) for _ in range(3)] for a in q]
    want = []
    for i in range(3):
        for a, x in zip(q, sources):
            a.x.copy_(x[i])
            a.run()
        torch.cuda.synchronize()
        want.append([a.results() for a in q])
    graphs = []
    for a, t in zip(q, s):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(t), torch.cuda.graph(graphs[-1], stream=t):
            a.run(torch.cuda.current_stream())
    for i in (2, 0, 1):
        for a, x in zip(q, sources):
            a.x.copy_(x[i])
        torch.cuda.synchronize()
        for _ in range(2):
            for g, t in zip(graphs, s):  # side by side
                with torch.cuda.stream(t):
                    g.replay()
        torch.cuda.synchronize()
        for a, w in zip(q, want[i]):
            assert all(torch.equal(x, y) for x, y in zip(a.results(), w)), i
    for i in range(3):
        for a, x in zip(q, sources):
            a.x.copy_(x[i])
        torch.cuda.synchronize()
        for a, t in zip(q, s):
            a.run(t)
        torch.cuda.synchronize()
        for a, w in zip(q, want[i]):
            assert all(torch.equal(x, y) for x, y in zip(a.results(), w)), i
    assert lib[0].cb_linear_device_status() == 0
    for a in q:
        a.close()


def test_rows_far_apart(lib):
    """Rows of codes, results and outputs in 4 bits that begin behind 2^32 bytes."""
    block, cb = lib
    m, n, k, stride = 40, 96, 128, 1 << 28  # elements: a row of codes every 128 MB
    rng = np.random.default_rng(2)
    v, u = rng.standard_normal((m, k)), rng.standard_normal((n, k))
    held, codes, tiles = R.quantised(v)
    wheld, wcodes, wtiles = R.quantised(u)
    buf = torch.zeros(m, stride // 2, dtype=torch.uint8, device="cuda")
    buf[:, :k // 2] = torch.from_numpy(codes).cuda()
    x_scale, w, w_scale = (torch.from_numpy(t).cuda() for t in (tiles, wcodes, wtiles))
    out = torch.zeros(m, 1 << 26, dtype=torch.float32, device="cuda")
    layer = block.cb_linear_create(w, n, k, cb.CB_MXFP4, w_scale)
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, x_stride=stride, out_stride=1 << 26, out_dtype=cb.CB_FP32), buf, x_scale, out=out)
    torch.cuda.synchronize()
    want = torch.from_numpy(held @ wheld.T)
    bound = (k + 4) * U * torch.from_numpy(np.abs(held) @ np.abs(wheld).T)
    assert bool(((out[:, :n].double().cpu() - want).abs() <= bound).all()) and float(out[:, n:n + 64].abs().max()) == 0.0
    del out
    mx, scale = torch.zeros(m, stride // 2, dtype=torch.uint8, device="cuda"), torch.zeros(block.cb_mx_scale_bytes(m, n), dtype=torch.uint8, device="cuda")
    io = block.cb_linear_io(rows=m, x_stride=stride, out_stride=stride, out_dtype=cb.CB_MXFP4, out_scale=scale.data_ptr())
    block.cb_linear_run(layer, io, buf, x_scale, out=mx)
    torch.cuda.synchronize()
    R.check_quantised(want.numpy(), bound.numpy(), mx[:, :n // 2].cpu().numpy(), scale.cpu().numpy(), 0)
    assert int(mx[:, n // 2:n].max()) == 0
    block.cb_linear_destroy(layer)


# single tiles and several a CTA, single CTAs and pairs; outputs in bf16, fp32 and 4 bits, hidden states by TMA for short and long sums, results off the grid;
# parts of K, passes
@pytest.mark.parametrize("m,n,k,out,resid", [(40, 64, 64, "bf16", False), (8, 64, 64, "bf16", False), (4096, 4608, 512, "bf16", False),
                                             (4096, 4608, 512, "mx", False), (3000, 2000, 512, None, True), (3000, 2000, 8192, "bf16", True),
                                             (500, 333, 264, "bf16", True), (77, 1152, 8192, "bf16", False), (1000, 1000, 20000, "fp32", False)])
def test_a_wait_that_runs_out(lib, m, n, k, out, resid):
    block, cb = lib
    rng = np.random.default_rng(m)
    v, u = rng.integers(-2, 3, (m, k)).astype(float), rng.integers(-2, 3, (n, k)).astype(float)
    v[:, ::32] = 2.0  # a power of two of 1/2 for each block: codes of 4, and sums of whole numbers
    u[:, 16:] = 0.0
    u[:, 0] = 2.0
    (xv, xc, xs), (wv, wc, ws) = R.quantised(v), R.quantised(u)
    xc, xs, wc, ws = (torch.from_numpy(t).cuda() for t in (xc, xs, wc, ws))
    assert np.array_equal(xv, v) and np.array_equal(wv, u)
    ref = torch.from_numpy(v[:, :16] @ u[:, :16].T)
    mx = out == "mx"
    y = torch.zeros(m, n, device="cuda", dtype=torch.float32 if out == "fp32" else torch.bfloat16) if out else None
    if mx:
        y = torch.zeros(m, -(-n // 32) * 16, device="cuda", dtype=torch.uint8)
    scale = torch.zeros(block.cb_mx_scale_bytes(m, n), dtype=torch.uint8, device="cuda")
    r = torch.randint(-2, 3, (m, n), device="cuda").bfloat16() if resid else None
    xo = torch.zeros_like(r) if resid else None
    layer = block.cb_linear_create(wc, n, k, cb.CB_MXFP4, ws)
    io = block.cb_linear_io(rows=m, out_dtype=cb.CB_MXFP4 if mx else cb.CB_FP32 if out == "fp32" else cb.CB_BF16, resid_dtype=cb.CB_BF16,
                            out_scale=scale.data_ptr())
    assert block.cb_linear_device_status() == 0
    for turn in range(2):
        block.cb_linear_set_option(layer, cb.CB_OPT_WAIT_NS, 20_000_000)
        block.cb_linear_set_option(layer, cb.CB_OPT_TEST_WITHHOLD, 1)
        t0 = time.perf_counter()
        block.cb_linear_run(layer, io, xc, xs, resid=r, out=y, resid_out=xo)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 5.0
        assert block.cb_linear_device_status() & cb.CB_DEV_CONSUMER_TIMEOUT
        assert block.cb_linear_device_status() == 0  # the read cleared it
        block.cb_linear_set_option(layer, cb.CB_OPT_TEST_WITHHOLD, 0)
        block.cb_linear_set_option(layer, cb.CB_OPT_WAIT_NS, 10 ** 9)
        block.cb_linear_run(layer, io, xc, xs, resid=r, out=y, resid_out=xo)
        torch.cuda.synchronize()
        assert block.cb_linear_device_status() == 0
        if mx:
            R.check_quantised(ref.numpy(), np.zeros((m, n)), y.cpu().numpy(), scale.cpu().numpy(), 0)
        elif y is not None:
            assert torch.equal(y.cpu().double(), ref)
        assert xo is None or torch.equal(xo.cpu().double(), r.cpu().double() + ref)
    block.cb_linear_destroy(layer)
