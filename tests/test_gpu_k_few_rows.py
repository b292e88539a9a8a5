"""cb_linear_run for up to 32 rows whose last bytes do not fill a piece of 16: rows on 16-byte boundaries, of every length within a turn of 64 bytes,
with NaN before, between and behind them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def rows_of(rows, k, type, g):
    """Whole numbers from -4 to 4, the last row's end followed by NaN at once."""
    stride = (k + 15) // 16 * 16
    buf = torch.full((64 + rows * stride + 64,), float("nan"), device="cuda").to(DT[type])
    v = torch.as_strided(buf, (rows, k), (stride, 1), 64)
    v.copy_(torch.randint(-4, 5, (rows, k), generator=g, device="cuda").to(DT[type]))
    return v, stride


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("m,n", [(1, 1), (8, 40), (9, 17), (32, 100), (5, 3700)])
def test_rows_that_end_inside_a_piece(lib, type, m, n):
    block, cb = lib
    g = torch.Generator(device="cuda").manual_seed(m)
    for k in (*range(1, 68), 127, 129, 1000, 1023, 1025, 2047, 4097, 4104, 8191):
        (x, xs), (w, ws) = rows_of(m, k, type, g), rows_of(n, k, type, g)
        y = torch.empty(m, n, device="cuda")
        layer = block.cb_linear_create(w, n, k, cb.CB_BF16 if type == "bf16" else cb.CB_E4M3, w_stride=ws)
        block.cb_linear_run(layer, block.cb_linear_io(rows=m, x_stride=xs, out_dtype=cb.CB_FP32), x, out=y)
        assert torch.equal(y.double(), x.float().double() @ w.float().double().t()), k  # exact: sums below 2^24
        block.cb_linear_destroy(layer)
