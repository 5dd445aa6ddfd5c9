"""The torch side of the gated recurrence and the orthogonalised update: autograd through the
sequence against autograd through the formulas, and the example end to end."""
import importlib.util
import os

import pytest
import torch

from paper_2609_13716_gb300 import recurrent

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def formulas(x, r, i, lam, h0, reset):
    s = 8 * torch.nn.functional.softplus(lam)
    a = torch.exp(-s * torch.sigmoid(r))
    b = torch.sqrt(1 - a * a) * torch.sigmoid(i) * x
    keep = (1 - reset.double())[..., None]
    y, out = h0, []
    for t in range(x.shape[0]):
        y = keep[t] * a[t] * y + b[t]
        out.append(y)
    return torch.stack(out), y


def test_autograd_matches_the_formulas():
    """fp32 gradients of a nonlinear loss against fp64 autograd; 5e-5 of each gradient's norm
    (fp32 roundings of the forward state enter the loss's own gradient: some 1e-6 each)."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    T, N, D = 30, 5, 48
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    proj, lam, h0 = rnd(T, N, 3 * D), rnd(D) - 4, rnd(N, D)
    reset = (torch.rand(T, N, device="cuda", generator=g) < 0.1).to(torch.uint8)
    grads = []
    for f64 in (False, True):
        leaves = [(v.double() if f64 else v.clone()).requires_grad_() for v in (proj, lam, h0)]
        x, r, i = leaves[0].split(D, dim=2)
        if f64:
            h, last = formulas(x, r, i, leaves[1], leaves[2], reset)
        else:
            h, last = recurrent.gated_recurrence(x, r, i, leaves[1], leaves[2], reset)
        loss = torch.tanh(h).square().sum() + (last ** 3).sum()
        loss.backward()
        grads.append([v.grad.double() for v in leaves])
    for a, b in zip(*grads):
        assert float((a - b).norm() / b.norm()) < 5e-5


def test_partial_gradients():
    """A loss of h alone, of the last state alone, and no gradient at all."""
    require_gpu()
    x, r, i = (torch.randn(9, 2, 32, device="cuda") for _ in range(3))
    lam = torch.full((32,), -4.0, device="cuda", requires_grad=True)
    for pick in (0, 1):
        out = recurrent.gated_recurrence(x, r, i, lam)
        lam.grad = None
        out[pick].sum().backward()
        assert torch.isfinite(lam.grad).all() and lam.grad.abs().sum() > 0
    with torch.no_grad():
        h, _ = recurrent.gated_recurrence(x, r, i, lam)
    assert not h.requires_grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_trains_and_serves(dtype):
    """The loss falls by a tenth at least, and single steps give the sequence's logits: bf16 h
    rounds the same way in both, fp32 differs by roundings (1e-3 of logits of order one)."""
    require_gpu()
    spec = importlib.util.spec_from_file_location("teammate_model", os.path.join(ROOT, "examples", "teammate_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, acc, gap = m.main(updates=25, envs=256, steps=48, dtype=dtype, verbose=False)
    assert losses[-1] < 0.9 * losses[0] and acc > 0.25
    assert gap < (1e-3 if dtype == "f32" else 0.1)
