"""Passes on both sides of the sizes where linear attention changes its form: chunks or steps by the width, the chains and the
steps of the last chunk; a warp or two a head.  Of many chains some are compared (test_gpu_linattn.py has the tolerances)."""
import pytest
import torch

import test_gpu_linattn as L

pytestmark = pytest.mark.gpu


def some_envs(T, N, H, K, V, dtype, seed=71):
    d = L.make(T, N, H, K, V, dtype, seed=seed, lengths=True)
    got = L.run(d)
    for n in sorted({0, N // 3, N - 1}):
        part = dict(d)
        for k in ("q", "k", "v", "do"):
            part[k] = d[k][:, n:n + 1]
        part["reset"], part["lengths"] = d["reset"][:, n:n + 1].contiguous(), d["lengths"][n:n + 1]
        part["s0"], part["ds_last"] = d["s0"][n:n + 1].contiguous(), d["ds_last"][n:n + 1].contiguous()
        L.verify({k: t[n:n + 1] if k in ("s_last", "ds0") else t[:, n:n + 1] for k, t in got.items()}, part)


@pytest.mark.parametrize("N,H,K,V,steps", [
    (3, 2, 64, 64, (5, 6, 7)), (320, 2, 64, 48, (9, 10, 11)), (100, 2, 32, 24, (11, 12, 13)), (310, 2, 32, 32, (19, 20, 21)),
    (20, 3, 16, 16, (23, 24, 25, 65)), (250, 4, 16, 12, (31, 32, 33, 64, 66)), (700, 2, 16, 16, (59, 60, 64, 65, 100, 119, 120, 129)),
    (2, 2, 100, 128, (2, 3)),
])
def test_chunks_or_steps(N, H, K, V, steps):
    for T in steps:
        some_envs(T, N, H, K, V, torch.bfloat16)


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("T,heads", [(4, 303), (4, 304), (9, 305), (63, 303), (64, 151), (64, 152), (96, 101), (96, 102), (1000, 9), (1000, 10),
                                     (61, 549), (61, 1100), (300, 34)])
@pytest.mark.parametrize("K,V", [(64, 64), (50, 33)])
def test_a_warp_or_two_a_head(T, heads, K, V, dtype):
    some_envs(T, heads, 1, K, V, dtype)
