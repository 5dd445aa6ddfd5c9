"""Host checks of the gated recurrence's entry points: they run before any CUDA call."""
import ctypes as C

import numpy as np
import pytest

import glr_ref as R


@pytest.fixture(scope="module")
def aht():
    from paper_2609_13716_gb300 import aht, build
    build.build()
    aht.load()
    return aht


def args(aht, **kw):
    s = aht.Seq(16, 8, 8)          # never dereferenced: every case below fails a host check
    d = dict(dtype=aht.AHT_FP32, D=8, T=4, N=2, x=s, r=s, i=s, lam=16, reset=None, lengths=None)
    d.update(kw)
    return aht.GlrArgs(*[d[k] for k, _ in aht.GlrArgs._fields_])


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=7), b"dtype"), (dict(D=0), b"sizes"), (dict(D=(1 << 20) + 1), b"sizes"), (dict(N=0), b"sizes"),
    (dict(T=-1), b"sizes"), (dict(N=1 << 40), b"2^37"), (dict(T=1 << 50), b"2^46"), (dict(lam=None), b"lam"),
])
def test_sizes_are_checked(aht, kw, word):
    L = aht.load()
    h = aht.Seq(16, 8, 8)
    a = args(aht, **kw)
    assert L.aht_glr_forward(C.byref(a), None, C.byref(h), None, None, None) == aht.AHT_EINVAL
    assert word in L.aht_last_error()
    assert L.aht_glr_backward(C.byref(a), 16, C.byref(h), None, C.byref(h), C.byref(h), C.byref(h), None, None, None,
                              0, None) == aht.AHT_EINVAL


def test_null_pointers_are_refused(aht):
    L = aht.load()
    h, none = aht.Seq(16, 8, 8), aht.Seq(None, 0, 0)
    a = args(aht)
    assert L.aht_glr_forward(None, None, C.byref(h), None, None, None) == aht.AHT_EINVAL
    assert L.aht_glr_forward(C.byref(a), None, C.byref(none), None, None, None) == aht.AHT_EINVAL
    for k in "xri":
        bad = args(aht, **{k: none})
        assert L.aht_glr_forward(C.byref(bad), None, C.byref(h), None, None, None) == aht.AHT_EINVAL
    back = lambda ck, *g, dlam=None, ws=None, n=0: L.aht_glr_backward(  # noqa: E731
        C.byref(a), ck, C.byref(h), None, *(C.byref(s) for s in g), dlam, None, ws, n, None)
    assert back(None, h, h, h) == aht.AHT_EINVAL
    assert back(16, h, none, h) == aht.AHT_EINVAL
    assert back(16, h, h, h, dlam=16) == aht.AHT_EINVAL
    assert back(16, h, h, h, dlam=16, ws=16, n=4) == aht.AHT_EINVAL and b"workspace" in L.aht_last_error()


def test_sizes_of_the_buffers(aht):
    assert aht.aht_glr_ckpt_shape(17, 3, 5) == (3, 3, 5)
    assert aht.load().aht_glr_ckpt_elems(17, 3, 5) == 45 and aht.load().aht_glr_ckpt_elems(0, 3, 5) == 0
    assert aht.load().aht_glr_ckpt_elems(-1, 3, 5) == 0 and aht.aht_glr_workspace(17, 3, 5) >= 60


def test_reference_gradient_is_the_forward_passes():
    """The 64-bit gradient against central differences of the 64-bit forward pass."""
    rng = np.random.default_rng(0)
    T, N, D = 11, 2, 3
    v = {k: rng.standard_normal((T, N, D)) for k in ("x", "r", "i")}
    lam, h0 = rng.standard_normal(D) - 3, rng.standard_normal((N, D))
    dh, dl = rng.standard_normal((T, N, D)), rng.standard_normal((N, D))
    reset, lens = (rng.random((T, N)) < 0.2), np.array([7, 11])

    def loss(x, r, i, lam, h0):
        h, last, _ = R.forward(x, r, i, lam, reset, lens, h0)
        return float((h * dh).sum() + (last * dl).sum())

    base = [v["x"], v["r"], v["i"], lam, h0]
    _, _, before = R.forward(*base[:4], reset, lens, h0)
    grads = R.backward(*base[:4], before, dh, reset, lens, dl)
    for k, g in enumerate(grads):
        u = rng.standard_normal(base[k].shape)
        up, dn = list(base), list(base)
        up[k], dn[k] = base[k] + 1e-5 * u, base[k] - 1e-5 * u
        assert abs((loss(*up) - loss(*dn)) / 2e-5 - (g * u).sum()) < 1e-6
