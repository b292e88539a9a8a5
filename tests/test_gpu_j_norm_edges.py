"""cb_norm_residual at its limits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_the_longest_row(lib, out):
    """2^31 - 1 elements, of which a thread has 2^22: the loops' indices end inside 32 bits. Ones, whose squares' sum is exact, behind
    which a guard stays as it is."""
    block, cb = lib
    n, guard = (1 << 31) - 1, 4096
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = torch.full((guard + n + guard,), 3.0, dtype=torch.bfloat16, device="cuda").to(torch.float8_e4m3fn if out == "e4m3" else torch.bfloat16)
    scale = torch.zeros(1, device="cuda") if out == "e4m3" else None
    desc = block.cb_norm_desc(rows=1, hidden=n, x_dtype=cb.CB_BF16, out_dtype=cb.CB_E4M3 if scale is not None else cb.CB_BF16, eps=0.0)
    block.cb_norm_residual(desc, x, x_out=x, out=y[guard:], out_scale=scale)
    torch.cuda.synchronize()
    want = 448.0 if out == "e4m3" else 1.0
    for i in range(0, n, 1 << 28):
        part = slice(i, min(i + (1 << 28), n))
        assert bool((y[guard:][part].bfloat16() == want).all()) and bool((x[part] == 1).all())
    assert bool((y[:guard].bfloat16() == 3).all()) and bool((y[guard + n:].bfloat16() == 3).all())
    if scale is not None:
        assert abs(float(scale) * 448 - 1) < 1e-6
