"""Calls whose tensors are not on the device that they run on are refused before anything is launched.
One GPU is enough: the current device, or the handle's, is given out as another one."""
import pytest
import torch

from paper_2609_13716_gb300 import aht, recurrent

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def sequences():
    x, r, i = (torch.randn(4, 3, 32, device="cuda") for _ in range(3))
    return x, r, i, torch.zeros(32, device="cuda")


def test_recurrence_on_another_current_device(monkeypatch):
    require_gpu()
    x, r, i, lam = sequences()
    h, ck = torch.full_like(x, 7.0), torch.empty(1, 3, 32, device="cuda")
    g = [torch.full_like(x, 7.0) for _ in range(3)]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    launched = []
    monkeypatch.setattr(aht, "load", lambda: launched.append(1))
    with pytest.raises(ValueError, match="cuda:0"):
        aht.aht_glr_forward(x, r, i, lam, h)
    with pytest.raises(ValueError, match="cuda:0"):
        aht.aht_glr_backward(x, r, i, lam, ck, x, *g)
    assert not launched


def test_optimiser_of_another_device():
    require_gpu()
    opt = aht.aht_muon_create([(8, 16)])
    assert opt.device == torch.cuda.current_device()
    w, m, g, o = (torch.ones(8, 16, device="cuda") for _ in range(4))
    opt.device += 1
    with pytest.raises(ValueError, match="cuda:0"):
        aht.aht_muon_step(opt, [w], [m], [g], 0.1)
    with pytest.raises(ValueError, match="cuda:0"):
        aht.aht_muon_orthogonalize(opt, [g], [o])
    opt.device -= 1
    aht.aht_muon_orthogonalize(opt, [g], [o])
    aht.aht_muon_sync(opt)
    assert (w == 1).all() and (m == 1).all()
    opt.close()


def test_torch_side_makes_the_tensors_device_current(monkeypatch):
    """With another device current, the tensors' own is while the library is called, and not after."""
    require_gpu()
    x, r, i, lam = sequences()
    p = torch.nn.Parameter(torch.ones(8, 16, device="cuda"))
    current, entered = [1], []

    class Guard:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            entered.append(self.index)
            self.before, current[0] = current[0], self.index

        def __exit__(self, *a):
            current[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    x.requires_grad_()
    h, last = recurrent.gated_recurrence(x, r, i, lam)
    h.sum().backward()
    recurrent.gated_step(x[0].detach(), r[0], i[0], lam, torch.zeros(3, 32, device="cuda:0"))
    opt = recurrent.OrthogonalOptimizer([p])
    assert entered == [0] * 4 and current == [1] and opt.handle.device == 0
    current[0] = 0                             # the tensors' device is current: nothing to enter
    recurrent.gated_step(x[0].detach(), r[0], i[0], lam, torch.zeros(3, 32, device="cuda:0"))
    assert entered == [0] * 4


def test_host_tensors_are_still_a_type_error():
    require_gpu()
    x, r, i, lam = sequences()
    h = torch.empty_like(x)
    for bad in ((x.cpu(), r, i, lam), (x, r.cpu(), i, lam), (x, r, i, lam.cpu())):
        with pytest.raises(TypeError, match="CUDA"):
            aht.aht_glr_forward(*bad, h)
    with pytest.raises(TypeError, match="CUDA"):
        aht.aht_glr_forward(x, r, i, lam, h, h0=torch.zeros(3, 32))
