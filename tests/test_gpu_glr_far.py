"""Rows whose element offsets pass 2^31, inputs, states and gradients alike: the stores of both passes,
whole chains and passes split over a cluster, against the same call on dense tensors.  Aligned views run
the same kernels (the same bits); others are compared with the tolerances of test_gpu_glr.py."""
import pytest
import torch

from gpu_util import np_, require_gpu
from paper_2609_13716_gb300 import aht
from test_gpu_glr import bwd, fwd, near, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,st,sn", [
    (3, 2, 64, 1_500_000_000, 700_000_000),          # whole chains
    (3, 2, 64, 1_500_000_001, 700_000_003),
    (1100, 2, 64, 2_800_000, 1_400_000),             # split over a cluster
    (1100, 2, 64, 2_800_001, 1_400_003),
    (2, 3, 64, 64, 1_600_000_000),                   # env-major
])
def test_far_views(T, N, D, st, sn, dtype):
    require_gpu()
    need = (T - 1) * st + (N - 1) * sn + 20_000
    esz = 4 if dtype == "f32" else 2
    if torch.cuda.mem_get_info()[0] < need * esz + (8 << 30):
        pytest.skip("needs %d GB" % (need * esz >> 30))
    assert (T - 1) * st + (N - 1) * sn > 1 << 31
    p = problem(T, N, D, dtype, resets=0.01)
    h0, l0, c0 = fwd(p)
    want = dict(bwd(p, c0), h=h0, h_last=l0)
    big = torch.empty(need, dtype=p["x"].dtype, device="cuda")
    view = {k: torch.as_strided(big, (T, N, D), (st, sn, 1), 1024 * n)
            for n, k in enumerate(("x", "r", "i", "dh", "h", "dx", "dr", "di"))}
    far = dict(p)
    for k in ("x", "r", "i", "dh"):
        view[k].copy_(p[k])
        far[k] = view[k]
    for k in ("h", "dx", "dr", "di"):
        view[k].fill_(float("nan"))
    _, l1, c1 = fwd(far, h=view["h"])
    dlam, dh0 = torch.empty(D, device="cuda"), torch.empty(N, D, device="cuda")
    ws = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device="cuda")
    aht.aht_glr_backward(far["x"], far["r"], far["i"], p["lam"], c1, far["dh"], view["dx"], view["dr"], view["di"], dlam, ws,
                         reset=p["reset"], dh_last=p["dh_last"], dh0=dh0)
    got = dict(h=view["h"], h_last=l1, dx=view["dx"], dr=view["dr"], di=view["di"], dlam=dlam, dh0=dh0)
    for k, v in want.items():
        if st % 8 == 0:
            assert torch.equal(got[k], v), k
        else:
            near(np_(got[k].float()), np_(v.float()), dtype if k in ("h", "dx", "dr", "di") else "f32", k)
    for k in ("x", "r", "i", "dh"):
        assert torch.equal(view[k], p[k]), k         # and nothing else was written
