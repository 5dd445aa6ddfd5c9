"""Views that begin at any element still run; addresses between elements are refused, and nothing is
written."""
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu
from test_gpu_glr import bwd, fwd, problem

pytestmark = pytest.mark.gpu


def test_a_workspace_between_floats():
    require_gpu()
    p = problem(8, 2, 16, "f32")
    _, _, ck = fwd(p)
    want = bwd(p, ck)
    n = aht.aht_glr_workspace(8, 2, 16)
    whole = torch.zeros(n + 16, dtype=torch.uint8, device="cuda")
    g = [torch.full_like(p["x"], 7.0) for _ in range(3)]
    dlam = torch.full((16,), 7.0, device="cuda")
    args = (p["x"], p["r"], p["i"], p["lam"], ck, p["dh"], *g, dlam)
    kw = dict(reset=p["reset"], dh_last=p["dh_last"])
    for off in (1, 2, 3):
        with pytest.raises(aht.AhtError) as e:
            aht.aht_glr_backward(*args, whole[off:off + n], **kw)
        assert e.value.status == aht.AHT_EINVAL
    assert all((t == 7.0).all() for t in [*g, dlam])
    aht.aht_glr_backward(*args, whole[4:4 + n], **kw)
    assert torch.equal(dlam, want["dlam"]) and torch.equal(g[0], want["dx"])


def between(t):
    """A tensor of the same values whose address lies one byte behind a multiple."""
    raw = torch.zeros(t.numel() * t.element_size() + 1, dtype=torch.uint8, device="cuda")
    return raw, raw.data_ptr() + 1


@pytest.mark.parametrize("which", ["W", "M", "G"])
def test_matrices_between_elements(which):
    require_gpu()
    import ctypes as C
    opt = aht.aht_muon_create([(8, 16)])
    t = {k: torch.ones(8, 16, device="cuda") for k in "WMG"}
    raw, at = between(t[which])
    ptr = {k: at if k == which else v.data_ptr() for k, v in t.items()}
    m = (aht.MuonMatrix * 1)(aht.MuonMatrix(ptr["W"], ptr["M"], ptr["G"], 16, 16, 16))
    L = aht.load()
    assert L.aht_muon_step(opt.handle, m, aht.AHT_FP32, 0.1) == aht.AHT_EINVAL and b"multiple" in L.aht_last_error()
    if which == "G":
        assert L.aht_muon_step(opt.handle, m, aht.AHT_BF16, 0.1) == aht.AHT_EINVAL
        one = (C.c_int32 * 1)(16)
        for a, b in ((at, t["W"].data_ptr()), (t["W"].data_ptr(), at)):
            for dt in (aht.AHT_FP32, aht.AHT_BF16):
                assert L.aht_muon_orthogonalize(opt.handle, (C.c_void_p * 1)(a), one, (C.c_void_p * 1)(b), one, dt) == aht.AHT_EINVAL
    aht.aht_muon_sync(opt)
    assert not raw.any() and all((v == 1).all() for v in t.values())
    opt.close()
