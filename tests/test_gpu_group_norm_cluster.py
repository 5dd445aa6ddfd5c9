"""Group norm of few long instances on a device that places no cluster of 16 CTAs: the reference and tolerances of
test_gpu_group_norm.py."""
import pytest
import torch

from gpu_util import require_gpu
from paper_2609_13716_gb300 import aht
from test_gpu_group_norm import check, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[8, 16])
def most(request):
    require_gpu()
    aht.aht_debug_group_norm_cluster(request.param)
    yield request.param
    aht.aht_debug_group_norm_cluster(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,L,C,G", [(1, 60000, 16, 1), (1, 400000, 8, 1), (4, 70001, 10, 2), (1, 30000, 40, 8)])
def test_few_long_instances(N, L, C, G, dtype, most):
    check(make(N, L, C, dtype, seed=51, lengths=N > 2), G, "silu")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_channels_of_many_vectors(dtype, most):
    """More vectors a position than threads: dweight and dbias come from a pass of their own."""
    check(make(1, 600, 8192, dtype, seed=52), 1, "none")


def test_what_the_device_says():
    """A whole GPU places clusters of 16: asked, the call gives their bits."""
    require_gpu()
    d = make(1, 200000, 24, torch.bfloat16, seed=53)
    asked = run(d, 1, "silu")
    aht.aht_debug_group_norm_cluster(16)
    try:
        wide = run(d, 1, "silu")
    finally:
        aht.aht_debug_group_norm_cluster(0)
    assert all(torch.equal(asked[n], wide[n]) for n in asked)
