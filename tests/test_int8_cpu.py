"""Host side of the int8 history: its layout, and what a plan of that type refuses."""
import pytest


@pytest.fixture(scope="module")
def cb():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import chebboost
    return chebboost


def test_cache_layout(cb):
    numels = [1, 63, 64, 65, 256, 257, 8192, 8193, 100000]
    for K in (1, 3, 8):
        p = cb.cb_plan_create([9.0 - k for k in range(K)], K, [(i, 0, n, -1) for i, n in enumerate(numels)], cb.CB_INT8, 0.0, 9.0)
        slot = sum((n + 255) // 256 * 256 + (2 * ((n + 63) // 64) + 255) // 256 * 256 for n in numels)
        assert cb.cb_plan_cache_bytes(p) == K * slot + cb.CB_STATUS_BYTES
        with pytest.raises(cb.CbError) as e:
            cb.cb_plan_bind_cache(p, 0x1000, K * slot + cb.CB_STATUS_BYTES - 1)
        assert e.value.status == cb.CB_ERR_ARG
        cb.cb_plan_destroy(p)


@pytest.mark.parametrize("dtype", [3, 4, -1])
def test_other_cache_types_are_refused(cb, dtype):
    with pytest.raises(cb.CbError) as e:
        cb.cb_plan_create([2.0, 1.0], 2, [(0, 0, 8, -1)], dtype, 0.0, 2.0)
    assert e.value.status == cb.CB_ERR_ARG


def test_largest_tensor_has_a_slot_size(cb):
    p = cb.cb_plan_create([2.0, 1.0], 2, [(0, 0, cb.CB_MAX_NUMEL, -1)], cb.CB_INT8, 0.0, 2.0)
    assert cb.cb_plan_cache_bytes(p) == 2 * (cb.CB_MAX_NUMEL + cb.CB_MAX_NUMEL // 32) + cb.CB_STATUS_BYTES
    cb.cb_plan_destroy(p)
