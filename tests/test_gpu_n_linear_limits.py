"""Waits of cb_linear_run's kernels that run out: operands of which more is announced than is copied. The kernel notes it in the status word and
returns; what shared memory and TMEM it held is free again, and the next call is right."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


# a single tile and several a CTA, single CTAs and pairs, in bf16 and e4m3; an output, a hidden state and both by TMA, results off the grid; parts of K, passes
@pytest.mark.parametrize("type", ["bf16", "e4m3"])
@pytest.mark.parametrize("m,n,k,out,resid", [(40, 64, 64, "bf16", False), (4096, 4608, 256, "bf16", False), (3000, 2000, 512, None, True),
                                             (3000, 2000, 512, "fp32", True), (500, 333, 264, "bf16", True), (77, 1152, 4096, "bf16", False),
                                             (1000, 1000, 8192, "fp32", False)])
def test_a_wait_that_runs_out(lib, type, m, n, k, out, resid):
    block, cb = lib
    dt = torch.bfloat16 if type == "bf16" else torch.float8_e4m3fn
    odt = torch.float32 if out == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(m)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda")  # noqa: E731
    x, w = whole(m, k).to(dt), whole(n, k)
    w[:, 16:] = 0  # sums of up to 64, exact in every type
    w = w.to(dt)
    y = torch.zeros(m, n, device="cuda", dtype=odt) if out else None
    r = whole(m, n).bfloat16() if resid else None
    xo = torch.zeros_like(r) if resid else None
    ref = x.float() @ w.float().t()
    layer = block.cb_linear_create(w, n, k, cb.CB_BF16 if type == "bf16" else cb.CB_E4M3)
    io = block.cb_linear_io(rows=m, out_dtype=cb.CB_FP32 if out == "fp32" else cb.CB_BF16, resid_dtype=cb.CB_BF16)
    assert block.cb_linear_device_status() == 0
    for turn in range(2):
        block.cb_linear_set_option(layer, cb.CB_OPT_WAIT_NS, 20_000_000)
        block.cb_linear_set_option(layer, cb.CB_OPT_TEST_WITHHOLD, 1)
        t0 = time.perf_counter()
        block.cb_linear_run(layer, io, x, resid=r, out=y, resid_out=xo)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 5.0
        assert block.cb_linear_device_status() & cb.CB_DEV_CONSUMER_TIMEOUT
        assert block.cb_linear_device_status() == 0  # the read cleared it
        block.cb_linear_set_option(layer, cb.CB_OPT_TEST_WITHHOLD, 0)
        block.cb_linear_set_option(layer, cb.CB_OPT_WAIT_NS, 10 ** 9)
        block.cb_linear_run(layer, io, x, resid=r, out=y, resid_out=xo)
        torch.cuda.synchronize()
        assert block.cb_linear_device_status() == 0
        assert y is None or torch.equal(y.float(), ref)
        assert xo is None or torch.equal(xo.float(), r.float() + ref)
    block.cb_linear_destroy(layer)


def test_options_out_of_range_are_refused(lib):
    block, cb = lib
    w = torch.zeros(8, 8, device="cuda").bfloat16()
    layer = block.cb_linear_create(w, 8, 8, cb.CB_BF16)
    for option, value in ((cb.CB_OPT_WAIT_NS, -1), (cb.CB_OPT_WAIT_NS, 6 * 10 ** 10 + 1), (cb.CB_OPT_TEST_WITHHOLD, 2), (cb.CB_OPT_KERNEL, 0)):
        with pytest.raises(cb.CbError) as e:
            block.cb_linear_set_option(layer, option, value)
        assert e.value.status == -1
    block.cb_linear_destroy(layer)
