"""What is not finite in a state, an input or a gradient goes where the formulas take it, however strong
the decay is and however the steps are split: only a reset drops it (test_gpu_glr.py)."""
import numpy as np
import pytest
import torch

from gpu_util import np_, require_gpu
from test_gpu_glr import bwd, fwd, problem
from test_gpu_glr_wide import reference

pytestmark = pytest.mark.gpu

SIZES = [(120, 1, 32), (128, 1, 32), (600, 1, 32), (1100, 3, 64), (2500, 1, 70),  # split: one CTA, clusters
         (40, 2000, 64), (19, 1830, 33), (1, 7, 64), (9, 3, 20)]                  # whole chains, one step
# lam = 0: the decay is 2^-4 a step, so 16 steps take it to 2^-64 and three such segments below fp32;
# lam = 60: one step takes it below fp32
LAM = [-4.0, 0.0, 60.0]


def patterns(p):
    h = torch.full_like(p["x"], 7.0)
    h, last, ck = fwd(p, h=h)
    got = dict(bwd(p, ck), h=h, h_last=last)
    return {k: np_(v.float()) for k, v in got.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["h0", "x first", "x middle", "r", "dh", "dh_last"])
@pytest.mark.parametrize("lam", LAM)
@pytest.mark.parametrize("T,N,D", SIZES)
def test_nan_comes_through(T, N, D, lam, where, dtype):
    require_gpu()
    p = problem(T, N, D, dtype, resets=0)
    p["lam"].fill_(lam)
    p["r"].zero_()
    bad = float("nan")
    if where == "h0":
        p["h0"][N // 2] = bad
    elif where == "x first":
        p["x"][0, N // 2] = bad
    elif where == "x middle":
        p["x"][T // 2, N // 2, 3:9] = bad
    elif where == "r":
        p["r"][T // 2, 0, 1] = bad
    elif where == "dh":
        p["dh"][T - 1, N // 2] = bad
    else:
        p["dh_last"][0, 5] = bad
    got, want = patterns(p), reference(p)
    for k, v in want.items():
        assert np.array_equal(np.isnan(got[k]), np.isnan(v)), k


@pytest.mark.parametrize("lam", LAM)
@pytest.mark.parametrize("T,N,D", SIZES)
def test_infinity_stays(T, N, D, lam):
    """An infinite state never decays, an infinite gradient of the last one reaches the first."""
    require_gpu()
    p = problem(T, N, D, "f32", resets=0)
    p["lam"].fill_(lam)
    p["r"].zero_()
    p["h0"][0, :4] = float("inf")
    p["h0"][0, 4:8] = float("-inf")
    p["dh_last"][0, 8:12] = float("-inf")
    got, want = patterns(p), reference(p)
    for k in ("h", "h_last", "dx", "di", "dh0"):
        assert np.array_equal(np.isposinf(got[k]), np.isposinf(want[k])), k
        assert np.array_equal(np.isneginf(got[k]), np.isneginf(want[k])), k
        assert np.array_equal(np.isnan(got[k]), np.isnan(want[k])), k
    assert np.array_equal(np.isfinite(got["dr"]), np.isfinite(want["dr"]))


@pytest.mark.parametrize("T,N,D", [(600, 1, 32), (2500, 2, 64), (40, 2000, 64)])
def test_a_reset_still_drops(T, N, D):
    """Resets between strong decays: the episode after one does not see NaN before it."""
    require_gpu()
    p = problem(T, N, D, "f32", resets=0)
    p["lam"].fill_(0.0)
    cut = T // 2
    p["reset"] = torch.zeros(T, N, dtype=torch.uint8, device="cuda")
    p["reset"][cut] = 1
    clean_h, clean_last, ck = fwd(p)
    clean = bwd(p, ck)
    p["h0"].fill_(float("nan"))
    p["dh"][cut] = float("nan")
    p["dh_last"].fill_(float("inf"))
    h, last, ck = fwd(p)
    got = bwd(p, ck)
    assert h[:cut].isnan().all() and torch.equal(h[cut:], clean_h[cut:]) and torch.equal(last, clean_last)
    assert torch.equal(got["dx"][:cut], clean["dx"][:cut]) and got["dx"][cut].isnan().all()
    assert torch.equal(got["dh0"], clean["dh0"])
