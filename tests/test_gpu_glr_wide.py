"""The gated recurrence where there are many envs (no split of the steps): every width of the
wide kernels, aligned and not, with resets and ragged lengths, against a reference in 64 bits
vectorised over the envs, on the rounded inputs.  Tolerances as in test_gpu_glr.py: fp32 results
2e-5 in the 2-norm and 4e-4 elementwise of max(rms, |value|), bf16 ones one rounding (4e-3)."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import np_, require_gpu
from test_gpu_glr import bwd, fwd, near, problem

pytestmark = pytest.mark.gpu


def reference(p):
    """Forward and backward in fp64 on the GPU, one step at a time."""
    f64 = torch.float64
    x, r, i, dh = (p[k].to(f64) for k in ("x", "r", "i", "dh"))
    T, N, D = x.shape
    lam = p["lam"].to(f64)
    soft = torch.log1p(torch.exp(-lam.abs())) + lam.clamp(min=0)
    rho, iota = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-i))
    q = 8 * soft * rho
    a, beta = torch.exp(-q), torch.sqrt(-torch.expm1(-2 * q))
    live = torch.ones(T, N, 1, dtype=torch.bool, device="cuda")
    if p["lengths"] is not None:
        live = (torch.arange(T, device="cuda")[:, None] < p["lengths"])[..., None]
    keep = torch.ones(T, N, 1, dtype=f64, device="cuda") if p["reset"] is None else 1 - p["reset"].to(f64)[..., None]
    decay = torch.where(live, a * keep, torch.ones_like(a))
    b = torch.where(live, beta * iota * x, torch.zeros_like(x))
    y, hs, before = p["h0"].to(f64), [], []
    for t in range(T):
        before.append(y)
        y = decay[t] * y + b[t]
        hs.append(y)
    h, before = torch.stack(hs), torch.stack(before)
    c, gs = p["dh_last"].to(f64), [None] * T
    for t in reversed(range(T)):
        gs[t] = torch.where(live[t], dh[t], torch.zeros_like(c)) + c
        c = decay[t] * gs[t]
    G = torch.where(live, torch.stack(gs), torch.zeros_like(h))
    dq = -a * (G * before * keep - G * iota * x * a / beta)
    out = dict(h=torch.where(live, h, torch.zeros_like(h)), h_last=y, dx=G * beta * iota,
               di=G * beta * x * iota * (1 - iota), dr=dq * q * (1 - rho),
               dlam=(dq * rho).sum((0, 1)) * 8 / (1 + torch.exp(-lam)), dh0=c)
    return {k: np_(v) for k, v in out.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,layout,ragged", [
    (37, 1900, 64, "time", False),       # two channels a thread, ring
    (21, 960, 128, "env", True),         # the same, env-major, ragged
    (40, 1850, 50, "time", False),       # two channels, rows not on 16 bytes
    (19, 1830, 33, "time", True),        # one channel
    (24, 700, 136, "fused", True),       # a last group of 8 channels; 512-aligned strides are not
])
def test_many_envs(T, N, D, layout, ragged, dtype):
    require_gpu()
    p = problem(T, N, D, dtype, layout, ragged=ragged)
    h, last, ck = fwd(p)
    got = dict(bwd(p, ck), h=h, h_last=last)
    for k, v in reference(p).items():
        near(np_(got[k].float()), v, dtype if k in ("h", "dx", "dr", "di") else "f32", k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,off", [(300, 100, 64, 0), (300, 100, 66, 0), (1100, 20, 64, 1), (700, 300, 48, 0), (2100, 3, 40, 0)])
def test_few_envs(T, N, D, off, dtype):
    """The steps split over warps and CTAs: aligned rows and views that begin off a boundary."""
    require_gpu()
    p = problem(T, N, D, dtype, ragged=N == 100)
    if off:
        for k in ("x", "r", "i", "dh"):
            w = torch.zeros(T, N, D + 3, dtype=p[k].dtype, device="cuda")
            w[:, :, off:off + D] = p[k]
            p[k] = w[:, :, off:off + D]
    h, last, ck = fwd(p, h=torch.full((T, N, D), float("nan"), dtype=p["x"].dtype, device="cuda"))
    got = dict(bwd(p, ck), h=h, h_last=last)
    for k, v in reference(p).items():
        near(np_(got[k].float()), v, dtype if k in ("h", "dx", "dr", "di") else "f32", k)


def test_offsets_beyond_32_bits():
    """Rows whose element offsets pass 2^31: a few steps and envs of a huge strided view."""
    require_gpu()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    T, N, D = 3, 2, 64
    p = problem(T, N, D, "bf16", resets=0)
    far = dict(p)
    big = torch.empty(T * 1_500_000_000, dtype=torch.bfloat16, device="cuda")
    for n, k in enumerate(("x", "r", "i", "dh")):   # steps 1.5e9 elements apart, envs 700e6
        v = torch.as_strided(big, (T, N, D), (1_500_000_000, 700_000_000, 1), 1000 * n)
        v.copy_(p[k])
        far[k] = v
    h0, l0, c0 = fwd(p)
    out = torch.as_strided(big, (T, N, D), (1_500_000_000, 700_000_000, 1), 8000)
    h1, l1, c1 = fwd(far, h=out)
    assert torch.equal(h0, h1) and torch.equal(l0, l1) and torch.equal(c0, c1)
    a, b = bwd(p, c0), bwd(dict(far, x=far["x"]), c1)
    for k in ("dlam", "dh0"):
        assert torch.equal(a[k], b[k])
