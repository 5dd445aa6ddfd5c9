"""A step lets go of its gradients while the update that reads them may still be waiting: their memory
is not handed out before, whichever stream they were allocated on."""
import pytest
import torch

from paper_2609_13716_gb300 import recurrent

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(512, 700), (128, 196)])
def test_memory_of_a_third_streams_gradient(shape):
    require_gpu()
    torch.manual_seed(0)
    w0, g = torch.randn(shape, device="cuda"), torch.randn(shape, device="cuda")
    made, filled, used = (torch.cuda.Stream() for _ in range(3))

    def run(own_streams):
        p = torch.nn.Parameter(w0.clone())
        torch.cuda.synchronize()
        with torch.cuda.stream(made):
            opt = recurrent.OrthogonalOptimizer([p], lr=0.05)
        torch.cuda.synchronize()
        a, b = (filled, used) if own_streams else (made, made)
        with torch.cuda.stream(a):
            p.grad = g.clone()
            held = p.grad.data_ptr()
        b.wait_stream(a)
        with torch.cuda.stream(b):
            torch.cuda._sleep(40_000_000)       # (clocks; about 20 ms)
            opt.step()
        with torch.cuda.stream(a):
            taken = [torch.full(shape, 1e6, device="cuda") for _ in range(3)]
        if own_streams:
            assert held not in [t.data_ptr() for t in taken]
        torch.cuda.synchronize()
        opt.sync()
        return p.detach().clone()

    assert torch.equal(run(False), run(True))
