"""cb_linear_run writes nothing behind a row's last feature: results whose rows start on 16-byte boundaries and end inside one are columns of a
wider tensor, or the last bytes of a buffer."""
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


def layer_of(lib, type, m, n, k):
    """A layer, its rows of x and their scales, and the plain product; whole numbers, exact in every type."""
    from paper_2608_23429_gb300 import mlp_branch as M
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(n)
    x, w = (torch.randint(-2, 3, (r, k), generator=g, device="cuda").float() for r in (m, n))
    w[:, 16:] = 0.0
    x[:, ::32], w[:, 0] = 2.0, 2.0
    if type == "mxfp4":
        held, wh = M.quantised(x), M.quantised(w)
        return block.cb_linear_create(wh[0], n, k, cb.CB_MXFP4, wh[1]), (*held, wh), x @ w.t()
    t = torch.bfloat16 if type == "bf16" else torch.float8_e4m3fn
    wt = w.to(t)
    return block.cb_linear_create(wt, n, k, cb.CB_BF16 if type == "bf16" else cb.CB_E4M3), (x.to(t), None, wt), x @ w.t()


@pytest.mark.parametrize("type", ["bf16", "e4m3", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n,wide", [(300, 260, 264), (300, 257, 264), (40, 262, 280), (4, 258, 264), (300, 264, 280), (1000, 301, 320)])
def test_columns_of_a_wider_tensor(lib, type, dtype, m, n, wide):
    block, cb = lib
    layer, (x, scale, _keep), want = layer_of(lib, type, m, n, 320)
    code = cb.CB_BF16 if dtype == "bf16" else cb.CB_FP32
    for out, resid in ((True, False), (False, True), (True, True)):
        y, r, xo = (torch.full((m, wide), v, dtype=DT[dtype], device="cuda") for v in (5.0, 6.0, 7.0))
        io = block.cb_linear_io(rows=m, out_stride=wide, resid_stride=wide, resid_out_stride=wide, out_dtype=code, resid_dtype=code)
        block.cb_linear_run(layer, io, x, scale, r if resid else None, None, y if out else None, xo if resid else None)
        torch.cuda.synchronize()
        assert bool((y[:, n:] == 5.0).all()) and bool((xo[:, n:] == 7.0).all())
        assert not out or torch.equal(y[:, :n].float(), want)
        assert not resid or torch.equal(xo[:, :n].float(), want + 6.0)
    assert block.cb_linear_device_status() == 0
    block.cb_linear_destroy(layer)


@pytest.mark.parametrize("type", ["bf16", "e4m3", "mxfp4"])
def test_the_last_row_ends_its_buffer(lib, type):
    """What lies behind the last row's last feature in the same allocation belongs to someone else."""
    block, cb = lib
    m, n, wide = 200, 260, 264
    layer, (x, scale, _keep), want = layer_of(lib, type, m, n, 320)
    buf = torch.full(((m - 1) * wide + n + 64,), 5.0, dtype=torch.bfloat16, device="cuda")
    block.cb_linear_run(layer, block.cb_linear_io(rows=m, out_stride=wide, out_dtype=cb.CB_BF16), x, scale, out=buf)
    torch.cuda.synchronize()
    assert bool((buf[(m - 1) * wide + n:] == 5.0).all())
    assert torch.equal(buf.as_strided((m, n), (wide, 1)).float(), want)
    block.cb_linear_destroy(layer)
