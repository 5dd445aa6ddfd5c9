"""A bounded wait of a split recurrence that runs out: the pass ends, what depends on the missing maps is
NaN, aht_glr_sync reports it, and the next pass is right.  The wait is made to run out on purpose
(aht_debug_glr_expire: an mbarrier nothing arrives on, a limit of some milliseconds)."""
import time

import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu
from test_gpu_glr import bwd, fwd, problem

pytestmark = pytest.mark.gpu

LIMIT = 5_000_000
SIZES = [(1100, 3, 64, "f32"), (1100, 3, 64, "bf16"), (700, 2, 35, "f32"), (5003, 1, 64, "bf16"), (300, 2, 32, "f32")]


@pytest.fixture(autouse=True)
def hook_off():
    yield
    aht.aht_debug_glr_expire(-1, 0)


def expired(call):
    t0 = time.monotonic()
    out = call()
    with pytest.raises(aht.AhtError) as e:
        aht.aht_glr_sync()
    assert e.value.status == aht.AHT_ETIMEOUT
    assert time.monotonic() - t0 < 5.0
    aht.aht_glr_sync()                 # reported once
    return out


@pytest.mark.parametrize("T,N,D,dtype,window", [(*s, 0) for s in SIZES] + [
    (5003, 1, 64, "bf16", 1), (5003, 1, 64, "f32", 2), (4500, 2, 35, "f32", 1)])   # (a window is up to 2048 steps)
def test_forward(T, N, D, dtype, window):
    require_gpu()
    p = problem(T, N, D, dtype, resets=0)
    want, last, ck = fwd(p)
    aht.aht_glr_sync()
    aht.aht_debug_glr_expire(window, LIMIT)
    h, l, _ = expired(lambda: fwd(p))
    assert l.isnan().all()
    bad = h.isnan()
    assert not bad[:1024 * window].any()                   # (the windows before it)
    assert bad.any() and torch.equal(h[~bad], want[~bad])  # NaN or right, nothing else
    again, l2, c2 = fwd(p)
    aht.aht_glr_sync()
    assert torch.equal(again, want) and torch.equal(l2, last) and torch.equal(c2, ck)


@pytest.mark.parametrize("T,N,D,dtype", SIZES)
def test_backward(T, N, D, dtype):
    require_gpu()
    p = problem(T, N, D, dtype, resets=0.01)
    _, _, ck = fwd(p)
    want = bwd(p, ck)
    aht.aht_glr_sync()
    aht.aht_debug_glr_expire(0, LIMIT)
    got = expired(lambda: bwd(p, ck))
    assert got["dh0"].isnan().all() and got["dlam"].isnan().all()
    for k in ("dx", "dr", "di"):
        bad = got[k].isnan()
        assert bad.any() and torch.equal(got[k][~bad], want[k][~bad]), k
    again = bwd(p, ck)
    aht.aht_glr_sync()
    for k, v in want.items():
        assert torch.equal(again[k], v), k


def test_the_hook_waits_for_a_split_pass():
    """Whole chains have no such wait; the hook stays set until a pass that has."""
    require_gpu()
    aht.aht_debug_glr_expire(0, LIMIT)
    wide = problem(20, 2000, 64, "f32")
    a, _, _ = fwd(wide)
    aht.aht_glr_sync()
    assert torch.isfinite(a).all()
    expired(lambda: fwd(problem(1100, 3, 64, "f32")))
    fwd(problem(1100, 3, 64, "f32"))
    aht.aht_glr_sync()
