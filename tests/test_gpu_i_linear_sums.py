"""What the sums and activations of cb_linear_run lose, where tolerances that follow the sums' sizes cannot see it, and its largest sizes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


def product(lib, x, w, out="fp32", act="NONE", rows=None):
    block, cb = lib
    code = {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32}
    layer = block.cb_linear_create(w, w.shape[0], w.shape[1], cb.CB_BF16 if w.dtype == torch.bfloat16 else cb.CB_E4M3,
                                   activation=getattr(block, "CB_ACT_" + act))
    y = torch.empty(x.shape[0], w.shape[0], device="cuda", dtype=DT[out])
    torch.cuda.synchronize()
    block.cb_linear_run(layer, block.cb_linear_io(rows=x.shape[0], out_dtype=code[out]), x, out=y)
    torch.cuda.synchronize()
    block.cb_linear_destroy(layer)
    assert block.cb_linear_device_status() == 0
    return y


# pre-activations on both sides of where the factor's denominator passes 2^30, and far beyond
TAIL = [0.0, -1.0, -4.0, -5.5, -5.6, -5.75, -6.0, -6.5, -8.0, -10.0, -12.5, -14.0, -20.0, -20.75, -21.0, -25.0, -30.0, -40.0, -60.0, -80.0, -87.0,
        -100.0, -1e3, -1e6, -1e9, -1e30, -3e38, 5.5, 20.0, 1e3, 1e9, 1e30, 3e38]


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["SILU", "GELU"])
@pytest.mark.parametrize("m,n,k", [(3, 33, 8), (40, 33, 8), (200, 264, 64), (40, 36, 8192)])  # few rows, off the grid, by TMA, parts of K
def test_activations_go_to_zero(lib, m, n, k, act, out):
    """One product of 1 with the value itself, so that sums are exact. With t the exponent (SiLU: -v, GELU: -2 sqrt(2/pi) (v +
    0.044715 v^3)), rounding t moves exp(t) by 3 u |t|, the remaining steps by 8 u: of the activation, not of the value. Below
    2^-126 the special function unit gives zero: 2^-126 |v|, taken up to where t passes 126 (v down to -88)."""
    v = torch.tensor(TAIL, dtype=torch.float32).bfloat16()
    x, w = torch.zeros(m, k, device="cuda").bfloat16(), torch.zeros(n, k, device="cuda").bfloat16()
    x[:, k - 3] = 1.0
    w[:, k - 3] = v.repeat(-(-n // len(TAIL)))[:n].cuda()
    y = product(lib, x, w, out, act).double()
    s = w[:, k - 3].double()
    t = -s if act == "SILU" else -2.0 * (2.0 / torch.pi) ** 0.5 * (s + 0.044715 * s ** 3)
    ref = s / (1.0 + torch.exp(t))
    slack = (16 + 4 * t.abs().clamp_max(200)) * U * ref.abs() + 2.0 ** -126 * 90
    step = ref.abs() * (2.0 ** -8 if out == "bf16" else 2.0 ** -24) + 2.0 ** -134  # half a step of the result, bf16's smallest included
    assert bool(((y - ref).abs() <= slack + step).all()), (s[((y - ref).abs() > slack + step).any(0)], y[0], ref)


@pytest.mark.parametrize("act", ["SILU", "GELU"])
@pytest.mark.parametrize("m,n", [(3, 40), (200, 40), (200, 33)])
def test_activations_of_values_that_are_not_finite(lib, m, n, act):
    """v / (1 + exp(-v)) and its like at the ends: NaN at -infinity (which it would divide by infinity), infinity at infinity; the
    values around them, which share a reciprocal with them, keep theirs but for its rounding (16 u, as above)."""
    x, w = torch.zeros(m, 64, device="cuda").bfloat16(), torch.zeros(n, 64, device="cuda").bfloat16()
    x[:, 0] = 1.0
    w[:, 0] = 1.5
    plain = product(lib, x, w, "fp32", act)[0, 0]
    for at, value in ((5, float("-inf")), (10, float("inf")), (15, float("nan"))):
        w[at, 0] = value
    y = product(lib, x, w, "fp32", act)
    assert bool(torch.isnan(y[:, 5]).all()) and bool((y[:, 10] == float("inf")).all()) and bool(torch.isnan(y[:, 15]).all())
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[[5, 10, 15]] = False
    assert bool(((y[:, rest] - plain).abs() <= 16 * U * plain).all())


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
def test_bf16_results_of_very_long_sums_are_not_cut_off(lib, type):
    """Positive terms, so that what a sum loses has one sign. Rounding to bf16 has none: over n results of a spread of more than a
    step its mean is off by 2^-9 / sqrt(n) at most, a tenth of the 2^-9 / 20 that the sums may lose."""
    m, n, k = 2048, 2048, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = (torch.empty(r, k, device="cuda", dtype=DT[type]) for r in (m, n))
    for t in (x, w):
        for i in range(0, t.shape[0], 256):
            t[i:i + 256] = (torch.rand(256, k, generator=g, device="cuda") * (0.5 + torch.rand(256, 1, generator=g, device="cuda"))).to(DT[type])
    y = product(lib, x, w, "bf16")[:256, :256].double()
    ref = sum(x[:256, i:i + 65536].float().double() @ w[:256, i:i + 65536].float().double().t() for i in range(0, k, 65536))
    off = float(((y - ref) / ref).mean())
    assert abs(off) < 2.0 ** -9 / 20, off


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("m,k", [(1, 4096), (8, 16384), (32, 16384), (1, 1 << 20), (32, 1 << 20)])
def test_fp32_sums_of_few_rows(lib, type, m, k):
    """As many output features as leave each row's sums to the warps of one CTA. A part of 512 products loses 1.3e-6 at most on the
    tensor cores (32 additions, each of which cuts off half of 2^-23 of a running sum that averages two thirds of the part's);
    the parts are then added rounded to nearest, which loses up to 2^-24 of the running sum each, independently: sqrt(parts) 2^-24."""
    n, seen = 3664, 64
    g = torch.Generator(device="cuda").manual_seed(k + m)
    for positive in (False, True):
        draw = lambda r: (torch.rand if positive else torch.randn)(r, k, generator=g, device="cuda").to(DT[type])  # noqa: E731
        x = draw(m)
        w = torch.empty(n, k, device="cuda", dtype=DT[type])
        for i in range(0, n, 229):  # (parts: memory for all of it in fp32 is not taken)
            w[i:i + 229] = draw(min(229, n - i))
        y = product(lib, x, w)[:, :seen].double()
        ref = sum(x[:, i:i + 65536].float().double() @ w[:seen, i:i + 65536].float().double().t() for i in range(0, k, 65536))
        off = float((y - ref).norm() / ref.norm())
        assert off < 1.3e-6 + (k / 512) ** 0.5 * U, off
        del x, w


@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("k", [4096, 16384, 1 << 17])
def test_fp32_sums_of_terms_of_one_sign(lib, type, k):
    """Over 32 rows, with the bound of test_fp32_sums_of_few_rows, and as many features as leave no parts of K to other tiles."""
    m, n, seen = 384, 12000, 64
    g = torch.Generator(device="cuda").manual_seed(k)
    x = torch.rand(m, k, generator=g, device="cuda").to(DT[type])
    w = torch.empty(n, k, device="cuda", dtype=DT[type])
    for i in range(0, n, 500):
        w[i:i + 500] = torch.rand(500, k, generator=g, device="cuda").to(DT[type])
    y = product(lib, x, w)[:, :seen].double()
    ref = sum(x[:, i:i + 16384].float().double() @ w[:seen, i:i + 16384].float().double().t() for i in range(0, k, 16384))
    off = float((y - ref).norm() / ref.norm())
    assert off < 1.3e-6 + (k / 512) ** 0.5 * U, off


def test_results_wider_than_2_31_bytes(lib):
    """Rows of fp32 results of 2^31 bytes and more, 76 GB in all."""
    m, n, k = 33, (1 << 29) + 1184, 8
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120e9:
        pytest.skip("needs 120 GB")
    x = torch.randint(-4, 5, (m, k), device="cuda").bfloat16()
    w = torch.randint(-4, 5, (n, k), device="cuda", dtype=torch.int8).bfloat16()
    y = product(lib, x, w)
    for at in (0, (1 << 28) - 512, (1 << 29) - 512, n - 1024):  # small whole numbers: exact
        assert torch.equal(y[:, at:at + 1024].double(), x.double() @ w[at:at + 1024].double().t())
    del y, w
    torch.cuda.empty_cache()
