"""The optimiser under streams other than the one it was made on."""
import pytest
import torch

from paper_2609_13716_gb300 import recurrent

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(64, 100), (300, 200)])
@pytest.mark.parametrize("made_on_side", [False, True])
def test_steps_follow_the_gradients_of_another_stream(shape, made_on_side):
    """Gradients that a busy stream fills late, an update there, weights read there: the same bits
    as on one stream."""
    require_gpu()
    torch.manual_seed(0)
    w0, grads = torch.randn(shape, device="cuda"), [torch.randn(shape, device="cuda") for _ in range(3)]

    def run(made, used):
        p = torch.nn.Parameter(w0.clone())
        torch.cuda.synchronize()
        with torch.cuda.stream(made):
            opt = recurrent.OrthogonalOptimizer([p], lr=0.05)
        torch.cuda.synchronize()
        out = []
        with torch.cuda.stream(used):
            for g in grads:
                p.grad = torch.zeros_like(p)
                torch.cuda._sleep(20_000_000)  # (clocks; about 10 ms)
                p.grad.copy_(g)
                opt.step()
                out.append(p.detach().clone())
        torch.cuda.synchronize()
        opt.sync()
        return out

    main, side = torch.cuda.default_stream(), torch.cuda.Stream()
    want = run(main, main)
    got = run(side, main) if made_on_side else run(main, side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
