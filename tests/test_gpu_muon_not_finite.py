"""NaN and infinity in some matrices of a set that runs products, where matrices share CTA pairs,
accumulators and exchange buffers (and once more on chip): the update of such a matrix is NaN as a whole,
and the others have the bits that they have beside finite ones."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu
from test_gpu_muon import gradient, padded

pytestmark = pytest.mark.gpu

SETS = [
    [(300, 260)] * 4,                                    # sums of three blocks: whole items
    [(1024, 1024), (300, 520), (100, 60)],               # shared items beside whole ones
    [(520, 700), (700, 520)],
    [(1024, 1024)] * 4 + [(1024, 128), (128, 196)],      # more items than pairs
    [(100, 140), (33, 700), (128, 128), (640, 90)],      # on chip
    [(1, 300), (300, 1), (1, 1), (200, 200)],            # sides of one
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("shapes", SETS)
def test_stays_in_its_matrix(shapes, bad, dtype):
    require_gpu()
    rng = np.random.default_rng(31)
    clean = [padded(gradient(rng, *s), dtype, pad=k % 3) for k, s in enumerate(shapes)]
    W0 = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in shapes]
    opt = aht.aht_muon_create(shapes)

    def update(grads):
        W, M = [w.clone() for w in W0], [torch.zeros(s, device="cuda") for s in shapes]
        aht.aht_muon_step(opt, W, M, grads, 0.1)
        aht.aht_muon_sync(opt)
        return W

    want = update(clean)
    for first in (0, 1):
        grads = [g.clone() for g in clean]
        hit = list(range(first, len(shapes), 2))
        for k in hit:
            r, c = shapes[k]
            grads[k][r // 2, c // 3] = bad
        got = update(grads)
        for k in range(len(shapes)):
            if k in hit:
                assert got[k].isnan().all(), (k, shapes[k])
            else:
                assert torch.equal(got[k], want[k]), (k, shapes[k])
    again = update(clean)
    assert all(torch.equal(a, b) for a, b in zip(again, want))
    opt.close()
