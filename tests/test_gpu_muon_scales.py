"""Orthogonalised updates of matrices whose entries' squares leave fp32's range, or whose norm does:
the factor does not depend on the scale.  Sets that run on chip and sets that run products, rows of
aligned groups and not, wide and tall.  Tolerances as in test_gpu_muon.py (bound_o)."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

import muon_ref as R
from gpu_util import np_, require_gpu
from test_gpu_muon import bound_o, gradient, off, padded

pytestmark = pytest.mark.gpu

SETS = [[(128, 196), (40, 96), (97, 50)], [(256, 300), (300, 129), (64, 77)]]
SCALES = [1e-41, 1e-30, 1e-25, 1e-19, 1e19, 1e25, 1e37]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("shapes", SETS)
def test_scale_of_the_entries(shapes, scale, dtype):
    require_gpu()
    eps = 1e-45 if scale < 1e-35 else 1e-38
    rng = np.random.default_rng(11)
    mats = [padded(gradient(rng, *s, scale=scale), dtype, pad=k) for k, s in enumerate(shapes)]
    outs = [torch.empty(s, dtype=m.dtype, device="cuda") for s, m in zip(shapes, mats)]
    opt = aht.aht_muon_create(shapes, eps=eps)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        assert torch.isfinite(m).all()
        ref = R.orthogonalize(np_(m.float()), eps=float(np.float32(eps)))
        assert off(o, ref) <= bound_o(ref, dtype), (m.shape, off(o, ref) / np.linalg.norm(ref))
    opt.close()


@pytest.mark.parametrize("big,rest", [(1e25, 1e-3), (1e-3, 1e-25), (1e30, 1e-30)])
@pytest.mark.parametrize("shapes", SETS)
def test_a_row_of_another_scale(shapes, big, rest):
    """One row far above all others: the others' squares are lost beside it, its own are not."""
    require_gpu()
    rng = np.random.default_rng(12)
    mats = []
    for k, s in enumerate(shapes):
        g = gradient(rng, *s, scale=rest)
        g[s[0] // 2] = gradient(rng, 1, s[1], scale=big)
        mats.append(padded(g, pad=k))
    outs = [torch.empty(s, device="cuda") for s in shapes]
    opt = aht.aht_muon_create(shapes, eps=1e-38)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        ref = R.orthogonalize(np_(m), eps=float(np.float32(1e-38)))
        assert off(o, ref) <= bound_o(ref), (m.shape, off(o, ref) / np.linalg.norm(ref))
    opt.close()


@pytest.mark.parametrize("scale", [1e-25, 1e25])
@pytest.mark.parametrize("shapes", SETS)
def test_update(shapes, scale):
    """W moves by the orthogonal factor whatever the gradient's scale; only a zero gradient has none."""
    require_gpu()
    rng = np.random.default_rng(13)
    G = [padded(gradient(rng, *s, scale=scale), pad=k) for k, s in enumerate(shapes)]
    W = [padded(rng.standard_normal(s).astype(np.float32), pad=k) for k, s in enumerate(shapes)]
    M = [torch.zeros(s, device="cuda") for s in shapes]
    W0 = [np_(w).astype(np.float64) for w in W]
    opt = aht.aht_muon_create(shapes, eps=1e-38)
    aht.aht_muon_step(opt, W, M, G, 0.1)
    aht.aht_muon_sync(opt)
    for k, s in enumerate(shapes):
        w, m, o = R.step(W0[k], np.zeros(s), np_(G[k]), 0.1, eps=float(np.float32(1e-38)))
        assert off(M[k], m) <= 2e-7 * np.linalg.norm(m)
        assert off(W[k], w) <= 2e-7 * np.linalg.norm(w) + 0.1 * np.sqrt(max(1, s[0] / s[1])) * bound_o(o)
    opt.close()
