"""Kernels of the recurrence that may start while the one before them drains still see all of its work:
inputs that arrive late on the stream, a chain of calls that feed one another, buffers written again
right after they were read, and the same captured into a graph."""
import pytest
import torch

from paper_2609_13716_gb300 import aht

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

SHAPES = [(64, 300, 128), (700, 3, 64), (1, 500, 128)]  # whole chains, split over a cluster, one step


def inputs(T, N, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return [rnd(T, N, D).to(dtype) for _ in range(3)] + [rnd(D) - 4]


def chain(x, r, i, lam, h, g, ckpt, ws, times=4):
    """Each pass reads the last one's h; the gradients read the last checkpoints."""
    for k in range(times):
        aht.aht_glr_forward(x if k == 0 else h[(k + 1) % 2], r, i, lam, h[k % 2], ckpt=ckpt)
    last = x if times == 1 else h[times % 2]
    dx, dr, di, dlam = g
    aht.aht_glr_backward(last, r, i, lam, ckpt, h[(times + 1) % 2], dx, dr, di, dlam, ws)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_late_inputs_and_chains(shape, dtype):
    require_gpu()
    T, N, D = shape
    x, r, i, lam = inputs(T, N, D, dtype)
    ckpt = torch.empty(aht.aht_glr_ckpt_shape(T, N, D), device="cuda")
    ws = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device="cuda")

    def buffers():
        return ([torch.empty_like(x) for _ in range(2)],
                [torch.empty_like(x) for _ in range(3)] + [torch.empty(D, device="cuda")])

    # every call waited for by the host
    h, g = buffers()
    for k in range(4):
        aht.aht_glr_forward(x if k == 0 else h[(k + 1) % 2], r, i, lam, h[k % 2], ckpt=ckpt)
        torch.cuda.synchronize()
    aht.aht_glr_backward(h[0], r, i, lam, ckpt, h[1], *g, ws)
    torch.cuda.synchronize()
    want = [*h, *g]

    late = [torch.full_like(t, float("nan")) for t in (x, r, i, lam)]
    h, g = buffers()
    torch.cuda._sleep(20_000_000)
    for a, b in zip(late, (x, r, i, lam)):
        a.copy_(b)
    chain(*late, h, g, ckpt, ws)
    for a in late:
        a.fill_(float("nan"))              # after the last reader, in the stream's order
    torch.cuda.synchronize()
    for a, b in zip([*h, *g], want):
        assert torch.equal(a, b)

    h, g = buffers()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for a, b in zip(late, (x, r, i, lam)):
            a.copy_(b)
        chain(*late, h, g, ckpt, ws)
        for a in late:
            a.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip([*h, *g], want):
        assert torch.equal(a, b)
