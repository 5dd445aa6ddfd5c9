"""What the torch side writes in place, autograd is told of: a graph that saved the earlier value refuses
to go backward, and one made afterwards uses the new value."""
import pytest
import torch

from paper_2609_13716_gb300 import recurrent

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(8, 16), (200, 150)])
def test_a_graph_from_before_an_update_is_refused(shape):
    require_gpu()
    torch.manual_seed(0)
    w = torch.nn.Parameter(torch.randn(shape, device="cuda"))
    opt = recurrent.OrthogonalOptimizer([w])
    x = torch.randn(5, shape[1], device="cuda", requires_grad=True)
    stale = (x @ w.t()).sum()                       # its gradient of x is w
    (x.detach() @ w.t()).square().sum().backward()
    before = w._version
    opt.step()
    assert w._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        stale.backward()
    (x @ w.t()).sum().backward()
    assert torch.allclose(x.grad, w.detach().sum(0).expand_as(x), rtol=1e-5, atol=1e-5)
    opt.sync()


def test_a_graph_from_before_a_step_is_refused():
    require_gpu()
    x, r, i = (torch.randn(4, 32, device="cuda") for _ in range(3))
    lam, state = torch.full((32,), -4.0, device="cuda"), torch.randn(4, 32, device="cuda")
    scale = torch.ones(32, device="cuda", requires_grad=True)
    stale = (scale * state).sum()                   # its gradient of scale is the state
    recurrent.gated_step(x, r, i, lam, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        stale.backward()
    (scale * state).sum().backward()
    assert torch.equal(scale.grad, state.sum(0))


def test_inference_tensors():
    """They have no version; a state made under inference_mode still serves, there and elsewhere."""
    require_gpu()
    lam = torch.full((32,), -4.0, device="cuda")
    with torch.inference_mode():
        x, r, i = (torch.randn(4, 32, device="cuda") for _ in range(3))
        state = torch.zeros(4, 32, device="cuda")
        a = recurrent.gated_step(x, r, i, lam, state)
    b = recurrent.gated_step(x, r, i, lam, state)
    assert torch.isfinite(a).all() and torch.isfinite(b).all() and state.abs().sum() > 0
