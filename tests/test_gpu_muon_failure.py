"""A bounded wait of an orthogonalised update that runs out: the call ends, aht_muon_sync reports it, what
is stored is as stated in include/aht.h, and the next call is right.  The wait is made to run out on
purpose (aht_debug_muon_expire: an mbarrier nothing arrives on, a limit of some milliseconds)."""
import time

import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu
from test_gpu_muon import gradient

pytestmark = pytest.mark.gpu

LIMIT = 5_000_000
ON_CHIP = [[(128, 196), (128, 128)], [(33, 20), (100, 900), (700, 64)], [(128, 1024)], [(20, 30)]]
PRODUCTS = [[(300, 200), (128, 640)], [(1024, 1024)],                        # shared sums
            [(128, 196), (1024, 128), (1024, 1024), (1024, 1024), (1024, 1024)]]  # more items than pairs


def arrays(shapes, seed=0):
    rng = np.random.default_rng(seed)
    up = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    return ([up(rng.standard_normal(s)) for s in shapes], [up(gradient(rng, *s)) for s in shapes],
            [up(gradient(rng, *s)) for s in shapes])


def clean(shapes):
    w, m, g = arrays(shapes)
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_step(opt, w, m, g, 0.1)
    aht.aht_muon_sync(opt)
    opt.close()
    return w, m


def expired(opt, w, m, g):
    t0 = time.monotonic()
    aht.aht_muon_step(opt, w, m, g, 0.1)
    with pytest.raises(aht.AhtError) as e:
        aht.aht_muon_sync(opt)
    assert e.value.status == aht.AHT_ETIMEOUT
    assert time.monotonic() - t0 < 5.0
    aht.aht_muon_sync(opt)             # reported once


def then_right(opt, shapes, want):
    w, m, g = arrays(shapes)
    aht.aht_muon_step(opt, w, m, g, 0.1)
    aht.aht_muon_sync(opt)
    for a, b in zip(w + m, want[0] + want[1]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("step", [0, 3, 4])
@pytest.mark.parametrize("shapes", ON_CHIP)
def test_on_chip(shapes, step):
    """No CTA of the matrix stores its columns; the other matrices are updated."""
    require_gpu()
    want = clean(shapes)
    bad = len(shapes) // 2
    opt = aht.aht_muon_create(shapes)
    w, m, g = arrays(shapes)
    before = w[bad].clone()
    aht.aht_debug_muon_expire(opt, bad, step, LIMIT)
    expired(opt, w, m, g)
    for k in range(len(shapes)):
        assert torch.equal(m[k], want[1][k])
        assert torch.equal(w[k], before if k == bad else want[0][k]), k
    then_right(opt, shapes, want)
    opt.close()


@pytest.mark.parametrize("step", [0, 3, 4])
@pytest.mark.parametrize("shapes", PRODUCTS)
def test_products(shapes, step):
    """The products stop before the last one of that matrix, so its weights are untouched."""
    require_gpu()
    want = clean(shapes)
    opt = aht.aht_muon_create(shapes)
    for bad in {0, len(shapes) - 1}:
        w, m, g = arrays(shapes)
        before = w[bad].clone()
        aht.aht_debug_muon_expire(opt, bad, step, LIMIT)
        expired(opt, w, m, g)
        assert torch.equal(w[bad], before)
        for a, b in zip(m, want[1]):
            assert torch.equal(a, b)
        then_right(opt, shapes, want)
    opt.close()


def test_the_hook_is_checked():
    require_gpu()
    opt = aht.aht_muon_create([(8, 16)], steps=2)
    for args in ((1, 0, LIMIT), (0, 2, LIMIT), (0, -1, LIMIT), (0, 0, 0), (0, 0, 1_000_000_001)):
        with pytest.raises(aht.AhtError) as e:
            aht.aht_debug_muon_expire(opt, *args)
        assert e.value.status == aht.AHT_EINVAL
    aht.aht_debug_muon_expire(opt, 0, 0, LIMIT)
    aht.aht_debug_muon_expire(opt, -1, 0, 0)
    out = torch.empty(8, 16, device="cuda")
    aht.aht_muon_orthogonalize(opt, [torch.ones(8, 16, device="cuda")], [out])
    aht.aht_muon_sync(opt)
    opt.close()
