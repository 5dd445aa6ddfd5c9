"""The gated recurrence where the decay leaves the neighbourhood of 1 (exponents s rho beyond 1/4): every
width of the whole-chain kernels, the split ones, one step, both types, against the formulas in 64 bits
on the rounded inputs (test_gpu_glr_wide.reference).

Tolerances, fixed before the first run.  A gate is about ten fp32 operations of 2^-24 relative error
each; the decay's exponent y = s rho log2 e is rounded once more, which moves a by 0.7 |y| 2^-24 of
itself, and what counts in a norm has |y| below 10 (a above 1e-3): together below 1e-6 of every
output but dlam in the 2-norm, as no channel here sums more than some tens of steps.  dlam is a sum of
terms of both signs over all steps and envs, so its own norm is smaller than its terms': as in
test_gpu_glr.py, 2e-5.  bf16 outputs round once more: 4e-3."""
import numpy as np
import pytest
import torch

from gpu_util import np_, require_gpu
from test_gpu_glr import bwd, fwd, near, problem
from test_gpu_glr_wide import reference

pytestmark = pytest.mark.gpu


def with_decay(p, kind):
    D = p["lam"].shape[0]
    if kind == "mixed":                      # per channel, from hardly any decay to nearly all
        lam = torch.linspace(-6, 6, D)
    elif kind == "groups":                   # warps that keep to the series beside warps that do not
        lam = torch.where(torch.arange(D) // 64 % 2 == 0, -5.0, 1.0)
    else:
        lam = torch.full((D,), float(kind))
    p["lam"] = lam.cuda()
    return p


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["-3", "0", "4", "8", "mixed", "groups"])
@pytest.mark.parametrize("T,N,D,layout,ragged", [
    (37, 1900, 64, "time", False),      # whole chains: two channels a thread, ring
    (21, 960, 128, "env", True),        # the same, env-major, ragged
    (30, 1850, 50, "time", True),       # two channels, rows not on 16 bytes
    (19, 1830, 33, "time", False),      # one channel
    (120, 5, 64, "fused", True),        # split over the warps of a CTA
    (1100, 3, 64, "time", True),        # over the CTAs of a cluster, ring
    (700, 3, 35, "time", False),        # the same, rows not on 16 bytes
    (1, 300, 128, "time", False),       # one step
    (1, 300, 33, "time", True),
])
def test_decay(T, N, D, layout, ragged, kind, dtype):
    require_gpu()
    p = with_decay(problem(T, N, D, dtype, layout, ragged=ragged), kind)
    h = torch.full((T, N, D), float("nan"), dtype=p["x"].dtype, device="cuda")
    h, last, ck = fwd(p, h=h)
    got = dict(bwd(p, ck), h=h, h_last=last)
    for k, v in reference(p).items():
        g = np_(got[k].float())
        near(g, v, dtype if k in ("h", "dx", "dr", "di") else "f32", k)
        if k != "dlam" and (dtype == "f32" or k in ("h_last", "dh0")):
            rel = np.linalg.norm(g - v) / np.linalg.norm(v)
            assert rel <= 1e-6, (k, rel)


@pytest.mark.parametrize("T,N,D", [(1, 40, 64), (200, 2, 64), (9, 2000, 64)])
def test_a_small_decay_is_as_accurate_as_a_large_one(T, N, D):
    """Fully open gates at s = 6, 12, 24 and 48, so a from 2e-3 to 1e-21: what the first step hands on (the
    state's share of h, by x = 0, and the initial state's gradient) is off by at most 4e-6 of each
    element: 0.7 |y| 2^-24 = 2.9e-6 at |y| = 69, and some roundings of s, a and the product."""
    require_gpu()
    p = problem(T, N, D, "f32", resets=0)
    s = torch.tensor([6.0, 12.0, 24.0, 48.0], dtype=torch.float64).repeat(D // 4)
    p["lam"] = torch.log(torch.expm1(s / 8)).float().cuda()
    p["r"].fill_(40.0)
    p["x"].zero_()
    p["dh_last"].zero_()
    h, last, ck = fwd(p)
    got = bwd(p, ck)
    lam = p["lam"].double()
    a = torch.exp(-8 * (torch.log1p(torch.exp(-lam.abs())) + lam.clamp(min=0)) / (1 + np.exp(-40.0)))
    want = a * p["h0"].double()
    assert float(((h[0].double() - want) / want).abs().max()) <= 4e-6
    g = torch.zeros(N, D, dtype=torch.float64, device="cuda")
    for t in reversed(range(T)):
        g = a * (p["dh"][t].double() + g)
    near_one = (g - got["dh0"].double()).abs() / g.abs()
    assert float(near_one.max()) <= 4e-6 + 1e-6      # (and the sum's rounding, where its terms cancel little)
