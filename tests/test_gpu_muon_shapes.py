"""Orthogonalised updates at the sizes between which the library chooses: matrices of a few hundred
rows, whose long sums two pairs of CTAs share and exchange, and sets that run a cluster of 1 to 8 CTAs
a matrix.  Against the formulas in 64 bits; the tolerances are test_gpu_muon's, which do not depend
on how a sum is divided."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

import muon_ref as R
from gpu_util import np_, require_gpu
from test_gpu_muon import bound_o, gradient, off, padded

pytestmark = pytest.mark.gpu

SHARED = [
    [(200, 600)],                          # only the first product's sum is long: 5 blocks, 3 + 2
    [(520, 700)],                          # an odd last row of blocks, 5 in every sum
    [(1000, 520), (100, 1100), (30, 20)],  # shared beside whole items; tall
    [(777, 130), (130, 777), (130, 777)],
    [(1024, 1024)],
    [(129, 4000)],                         # sums of 32 blocks and of 2
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", SHARED)
def test_shared_sums(shapes, dtype):
    require_gpu()
    rng = np.random.default_rng([len(shapes), *shapes[0]])
    mats = [padded(gradient(rng, *s), dtype, pad=2 * k) for k, s in enumerate(shapes)]
    outs = [padded(np.zeros(s, np.float32), dtype, pad=3 * k) for k, s in enumerate(shapes)]
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        ref = R.orthogonalize(np_(m.float()))
        assert off(o, ref) <= bound_o(ref, dtype), (m.shape, off(o, ref) / np.linalg.norm(ref))
    first = [o.clone() for o in outs]
    for _ in range(20):                    # calls back to back: the same sums in the same order
        aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for a, b in zip(first, outs):
        assert torch.equal(a, b)
    opt.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_update(dtype):
    """Two updates; every product of the first matrix is shared, the others' are not."""
    require_gpu()
    shapes = [(600, 760), (257, 130), (40, 300)]
    rng = np.random.default_rng(9)
    w = [padded(rng.standard_normal(s).astype(np.float32), pad=4) for s in shapes]
    m = [padded(np.zeros(s, np.float32), pad=1) for s in shapes]
    opt = aht.aht_muon_create(shapes)
    for _ in range(2):
        g = [padded(gradient(rng, *s), dtype, pad=2) for s in shapes]
        before = [(np_(a.clone()), np_(b.clone())) for a, b in zip(w, m)]
        aht.aht_muon_step(opt, w, m, g, 0.02)
        aht.aht_muon_sync(opt)
        for k, s in enumerate(shapes):
            ref, mom, o = R.step(*before[k], np_(g[k].float()), 0.02)
            scale = 0.02 * max(1.0, s[0] / s[1]) ** 0.5
            assert off(m[k], mom) <= 2e-7 * np.linalg.norm(mom)
            assert off(w[k], ref) <= scale * bound_o(o) + 2e-7 * np.linalg.norm(ref)
    opt.close()


@pytest.mark.parametrize("ctas", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("tall", [False, True])
def test_cluster_widths(ctas, tall):
    """A matrix that needs `ctas` CTAs, beside one that needs one; and a full last block."""
    require_gpu()
    long = 128 * ctas - (0 if ctas % 2 else 37)
    shapes = [(90 + ctas, long), (64, 33), (128, long)]
    shapes = [(c, r) if tall else (r, c) for r, c in shapes]
    rng = np.random.default_rng(20 + ctas)
    mats = [padded(gradient(rng, *s), pad=k) for k, s in enumerate(shapes)]
    outs = [padded(np.zeros(s, np.float32), pad=2 * k) for k, s in enumerate(shapes)]
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        ref = R.orthogonalize(np_(m))
        assert off(o, ref) <= bound_o(ref), (m.shape, off(o, ref) / np.linalg.norm(ref))
    opt.close()
