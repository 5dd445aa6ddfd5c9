"""Addresses that are no multiple of their elements' size, which a kernel must not be given: refused on the
host before any CUDA call."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def aht():
    from paper_2609_13716_gb300 import aht, build
    build.build()
    aht.load()
    return aht


def args(aht, dtype, **kw):
    s = aht.Seq(4096, 8, 8)          # never dereferenced: every case below fails a host check
    d = dict(dtype=dtype, D=8, T=4, N=2, x=s, r=s, i=s, lam=4096, reset=4097, lengths=None)
    d.update(kw)
    return aht.GlrArgs(*[d[k] for k, _ in aht.GlrArgs._fields_])


@pytest.mark.parametrize("name", ["x", "r", "i", "lam", "lengths", "h", "h0", "h_last", "ckpt"])
@pytest.mark.parametrize("dtype,off", [("AHT_FP32", 1), ("AHT_FP32", 2), ("AHT_BF16", 1)])
def test_forward(aht, dtype, off, name):
    L, code = aht.load(), getattr(aht, dtype)
    off = 2 if dtype == "AHT_BF16" and name not in "xrih" else off
    kw = {}
    if name in ("x", "r", "i"):
        kw[name] = aht.Seq(4096 + off, 8, 8)
    elif name in ("lam", "lengths"):
        kw[name] = 4096 + off
    other = {k: 4096 + (off if k == name else 0) for k in ("h", "h0", "h_last", "ckpt")}
    a, h = args(aht, code, **kw), aht.Seq(other["h"], 8, 8)
    assert L.aht_glr_forward(C.byref(a), other["h0"], C.byref(h), other["h_last"], other["ckpt"], None) == aht.AHT_EINVAL
    assert b"multiple" in L.aht_last_error()


@pytest.mark.parametrize("name", ["ckpt", "dh", "dh_last", "dx", "dr", "di", "dlam", "dh0", "ws"])
@pytest.mark.parametrize("dtype,off", [("AHT_FP32", 1), ("AHT_FP32", 2), ("AHT_BF16", 1)])
def test_backward(aht, dtype, off, name):
    L, code = aht.load(), getattr(aht, dtype)
    off = 2 if dtype == "AHT_BF16" and name in ("ckpt", "dh_last", "dlam", "dh0", "ws") else off
    at = {k: 4096 + (off if k == name else 0) for k in ("ckpt", "dh", "dh_last", "dx", "dr", "di", "dlam", "dh0", "ws")}
    seq = {k: aht.Seq(at[k], 8, 8) for k in ("dh", "dx", "dr", "di")}
    a = args(aht, code)
    assert L.aht_glr_backward(C.byref(a), at["ckpt"], C.byref(seq["dh"]), at["dh_last"], C.byref(seq["dx"]), C.byref(seq["dr"]),
                              C.byref(seq["di"]), at["dlam"], at["dh0"], at["ws"], 1 << 30, None) == aht.AHT_EINVAL
    assert b"multiple" in L.aht_last_error()
