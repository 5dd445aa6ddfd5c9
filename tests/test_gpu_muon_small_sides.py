"""Matrices with a short side of at most 32: the orthogonal factor is as accurate as the same iteration
with plain fp32 products.  Errors against 64 bits, root mean square over the matrices of a test.
The bound, fixed before the first run: 1.25 times the fp32 form's, the quarter for the spread of some
forty matrices' mean squares (each is within a factor of two of another)."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

import muon_ref as R
from gpu_util import np_, require_gpu

pytestmark = pytest.mark.gpu


def plain(u):
    x = u / (torch.sqrt((u * u).sum()) + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(5):
        g = x @ x.t()
        x = R.A * x + (R.B * g + R.C * (g @ g)) @ x
    return x.t() if tall else x


@pytest.mark.parametrize("beside", [None, (300, 200)])        # on chip, and in the products kernel
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("sides", [[(8, 8), (12, 12), (16, 16), (24, 24)], [(8, 32), (16, 64), (24, 96)]])
def test_as_accurate_as_fp32_products(sides, tall, beside):
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(21)
    shapes = [s[::-1] if tall else s for s in sides for _ in range(44 // len(sides))]
    mats = [torch.randn(s, device="cuda", generator=g) for s in shapes]
    if beside:
        shapes.append(beside)
        mats.append(torch.randn(beside, device="cuda", generator=g))
    outs = [torch.empty_like(m) for m in mats]
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    own, fp32 = [], []
    for m, o in list(zip(mats, outs))[:44 // len(sides) * len(sides)]:
        ref = R.orthogonalize(np_(m))
        for errors, got in ((own, o), (fp32, plain(m))):
            errors.append(np.linalg.norm(np_(got).astype(np.float64) - ref) / np.linalg.norm(ref))
    rms = [float(np.sqrt(np.mean(np.square(e)))) for e in (own, fp32)]
    assert rms[0] <= 1.25 * rms[1], rms
    opt.close()
