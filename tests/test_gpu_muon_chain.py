"""Calls of one handle that feed one another on the stream, without the host waiting in between: a
call's results are the next call's inputs, in either buffer and in place.  The same bits as with a
wait after every call."""
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

SETS = [[(128, 196), (128, 128)],            # on chip, a cluster of two
        [(100, 900), (33, 20), (700, 64)],   # on chip, a cluster of eight
        [(300, 200), (128, 640)]]            # products


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shapes", SETS)
def test_results_are_the_next_inputs(shapes, dtype):
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(len(shapes))
    first = [torch.randn(s, device="cuda", generator=g).to(dtype) for s in shapes]
    opt = aht.aht_muon_create(shapes, steps=2)

    def chain(wait):
        bufs = [[m.clone() for m in first], [torch.full_like(m, float("nan")) for m in first]]
        torch.cuda.synchronize()
        seen = []
        for k in range(8):
            src, dst = bufs[k % 2], bufs[(k + 1) % 2]
            aht.aht_muon_orthogonalize(opt, src, dst)
            if wait:
                torch.cuda.synchronize()
            aht.aht_muon_orthogonalize(opt, dst, dst)
            if wait:
                torch.cuda.synchronize()
                seen = [m.clone() for m in dst]
        torch.cuda.synchronize()
        return seen if wait else [m.clone() for m in dst]

    want = chain(True)
    for _ in range(20):
        for a, b in zip(want, chain(False)):
            assert torch.equal(a, b)
    aht.aht_muon_sync(opt)
    opt.close()


@pytest.mark.parametrize("shapes", SETS)
def test_updated_weights_are_the_next_gradients(shapes):
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(7)
    first = [torch.randn(s, device="cuda", generator=g) for s in shapes]
    opt = aht.aht_muon_create(shapes, steps=2)

    def chain(wait):
        a, b = [m.clone() for m in first], [m.flip(0).contiguous() for m in first]
        ma, mb = [torch.zeros_like(m) for m in first], [torch.zeros_like(m) for m in first]
        torch.cuda.synchronize()
        for _ in range(5):
            for w, m, grad in ((a, ma, b), (b, mb, a)):
                aht.aht_muon_step(opt, w, m, grad, 0.1)
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return a + b + ma + mb

    want = chain(True)
    for _ in range(10):
        for x, y in zip(want, chain(False)):
            assert torch.equal(x, y)
    aht.aht_muon_sync(opt)
    opt.close()
