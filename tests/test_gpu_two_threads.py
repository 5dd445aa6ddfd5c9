"""Two host threads that call the same kernels with different sizes at a time, each on a stream with buffers of its own:
every call succeeds, with the results of the calls made one after another.  The threads repeat the calls of the C ABI
that the binding makes, so that most of their time is in the library (where ctypes lets both run)."""
import threading

import pytest
import torch

from gpu_util import require_gpu
from paper_2609_13716_gb300 import aht

pytestmark = pytest.mark.gpu


class Calls:
    """Stands for the library and keeps the calls that the binding makes of it."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def keep(*args):
            self.made.append((name, args))
            return 0
        return keep


def norm(L, C, N, dtype, stream):
    """Instances that are kept in shared memory: its size goes with L."""
    torch.manual_seed(L)
    x, dy = (torch.randn(N, L, C, device="cuda").to(dtype) for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(2, N, 1, device="cuda")

    def call():
        aht.aht_group_norm_forward(x, 1, y, mean=mean, rstd=rstd, stream=stream)
        aht.aht_group_norm_backward(x, 1, mean, rstd, dy, dx, stream=stream)
    return call, (y, dx, x, dy, mean, rstd)


def loss(A, M, _, dtype, stream):
    torch.manual_seed(A)
    x, ref = (torch.randn(M, A, device="cuda").to(dtype) for _ in range(2))
    legal = torch.ones(M, A, device="cuda", dtype=torch.uint8)
    act, old, adv = torch.zeros(M, dtype=torch.int32, device="cuda"), torch.full((M,), -3.0, device="cuda"), torch.randn(M, device="cuda")
    stats, d = torch.empty(6, device="cuda"), torch.empty_like(x)
    ws = torch.empty(aht.aht_policy_loss_workspace(M, A), dtype=torch.uint8, device="cuda")

    def call():
        aht.aht_policy_loss(x, act, old, adv, stats, dlogits=d, legal=legal, ref_logits=ref, workspace=ws, kl_coef=0.1, stream=stream)
    return call, (stats, d, x, ref, legal, act, old, adv, ws)


@pytest.mark.parametrize("make,sizes,args", [
    (norm, (300, 1000), (64, 9, torch.float32)),
    (norm, (20000, 60000), (16, 1, torch.bfloat16)),
    (loss, (33, 64), (300, None, torch.float32)),
])
def test_sizes_of_two_threads(make, sizes, args, monkeypatch):
    require_gpu()
    lib = aht.load()
    streams = [torch.cuda.Stream() for _ in sizes]
    work = [make(n, *args, s) for n, s in zip(sizes, streams)]
    torch.cuda.synchronize()
    want, made = [], []
    for call, out in work:
        call()
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
        calls = Calls()
        with monkeypatch.context() as m:
            m.setattr(aht, "load", lambda: calls)
            call()
        made.append([(getattr(lib, name), a) for name, a in calls.made])
    failed = []

    def run(calls, stream):
        for i in range(20000):
            for f, a in calls:
                if f(*a):
                    failed.append((i, f.__name__))
                    return
            if i % 200 == 199:      # (not more than the launch queue holds)
                stream.synchronize()

    threads = [threading.Thread(target=run, args=a) for a in zip(made, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for (_, out), ref in zip(work, want):
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
