"""Host checks of the orthogonalised update's entry points: they run before any CUDA call."""
import ctypes as C

import numpy as np
import pytest

import muon_ref as R


@pytest.fixture(scope="module")
def aht():
    from paper_2609_13716_gb300 import aht, build
    build.build()
    aht.load()
    return aht


def create(aht, shapes, out=True, **cfg):
    c = dict(aht.MUON_DEFAULTS)
    c.update(cfg)
    n = len(shapes)
    h = C.c_void_p(99)
    st = aht.load().aht_muon_create(n, (C.c_int32 * n)(*[r for r, _ in shapes]), (C.c_int32 * n)(*[k for _, k in shapes]),
                                    C.byref(aht.MuonConfig(**c)), None, C.byref(h) if out else None)
    return st, h.value


@pytest.mark.parametrize("shapes,cfg,word", [
    ([], {}, b"MAX_MATRICES"), ([(4, 4)] * 49, {}, b"MAX_MATRICES"), ([(4, 0)], {}, b"MAX_DIM"), ([(16385, 4)], {}, b"MAX_DIM"),
    ([(4, 4)], dict(momentum=1.0), b"momentum"), ([(4, 4)], dict(momentum=float("nan")), b"momentum"),
    ([(4, 4)], dict(weight_decay=-0.1), b"weight_decay"), ([(4, 4)], dict(weight_decay=float("inf")), b"weight_decay"),
    ([(4, 4)], dict(eps=0.0), b"eps"), ([(4, 4)], dict(steps=0), b"steps"), ([(4, 4)], dict(steps=33), b"steps"),
])
def test_create_checks(aht, shapes, cfg, word):
    st, h = create(aht, shapes, **cfg)
    assert st == aht.AHT_EINVAL and h is None and word in aht.load().aht_last_error()


def test_null_arguments(aht):
    L = aht.load()
    h = C.c_void_p()
    one = (C.c_int32 * 1)(4)
    conf = aht.MuonConfig(**aht.MUON_DEFAULTS)
    assert L.aht_muon_create(1, one, one, C.byref(conf), None, None) == aht.AHT_EINVAL
    assert L.aht_muon_create(1, None, one, C.byref(conf), None, C.byref(h)) == aht.AHT_EINVAL
    assert L.aht_muon_create(1, one, one, None, None, C.byref(h)) == aht.AHT_EINVAL
    assert L.aht_muon_step(None, None, 0, 0.1) == aht.AHT_EINVAL
    assert L.aht_muon_orthogonalize(None, None, None, None, None, 0) == aht.AHT_EINVAL
    assert L.aht_muon_sync(None) == aht.AHT_EINVAL
    L.aht_muon_destroy(None)


def test_reference_singular_values():
    """The 64-bit reference maps each singular value by the quintic and keeps the vectors."""
    rng = np.random.default_rng(0)
    for shape in ((6, 9), (9, 6)):
        u = rng.standard_normal(shape)
        a, s, b = np.linalg.svd(u, full_matrices=False)
        s = s / np.sqrt((s * s).sum())
        for _ in range(5):
            s = R.A * s + R.B * s ** 3 + R.C * s ** 5
        assert np.allclose(R.orthogonalize(u, eps=0.0), (a * s) @ b, atol=1e-12)
        assert (s > 0.3).all() and (s < 1.21).all()


def test_singular_values_stay_bounded():
    """The bound the fp16 scales rest on: the quintic maps [0, 1.21] into itself, and the
    polynomial of the Gram matrix stays within [0, 3.4445] there."""
    s = np.linspace(0, 1.21, 200001)
    p = R.A * s + R.B * s ** 3 + R.C * s ** 5
    assert p.min() >= 0 and p.max() < 1.21
    q = R.A + R.B * s ** 2 + R.C * s ** 4
    assert q.min() > 0 and q.max() <= 3.4445 and 3.4445 * 8192 < 65504 and 1.21 ** 2 * 16384 < 65504
