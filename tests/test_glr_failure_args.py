"""Host checks of the recurrence's failure hook: they run before any CUDA call."""
import pytest


@pytest.fixture(scope="module")
def aht():
    from paper_2609_13716_gb300 import aht, build
    build.build()
    aht.load()
    return aht


def test_the_limit_is_checked(aht):
    L = aht.load()
    for bad in (0, -5, 1_000_000_001):
        assert L.aht_debug_glr_expire(0, bad) == aht.AHT_EINVAL and b"limit_ns" in L.aht_last_error()
    assert L.aht_debug_glr_expire(-1, 0) == aht.AHT_OK


def test_exported(aht):
    assert {"aht_glr_sync", "aht_debug_glr_expire"} <= set(aht.EXPORTED)
