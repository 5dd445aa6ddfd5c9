"""Orthogonalised matrix updates on the GPU (aht_muon_step, aht_muon_orthogonalize) against
the formulas in 64 bits (tests/muon_ref.py), on the rounded inputs.

Tolerances, fixed before the first run, in the 2-norm.  A step's operands carry 22 bits and
its products accumulate in fp32, so a step perturbs X by about 2^-21 ||X||_F; a perturbation
in a direction the input hardly has grows by at most 3.4445 per step, 3.4445^5 = 485 in all.
With ||X||_F = 1 at the start the orthogonal factor O is off by at most 485 * 2^-21 = 2.3e-4
in such directions, and by 2e-5 ||O|| (some tens of fp32 roundings) in those it has:
|O - ref| <= 2e-5 ||ref|| + 2.3e-4 in fp32, plus one rounding (2^-8 ||ref||) in bf16.  W adds
two fp32 roundings (2e-7 ||W||) to lr sqrt(max(1, rows / cols)) times that; M is one fused
multiply-add (2e-7)."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

import muon_ref as R
from gpu_util import np_, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def bound_o(ref, dtype="f32"):
    n = np.linalg.norm(ref)
    return 2e-5 * n + 485 * 2.0 ** -21 + (2.0 ** -8 * n if dtype == "bf16" else 0)


def off(got, ref):
    got = np_(got.float()).astype(np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all()
    return np.linalg.norm(got - ref)


def gradient(rng, r, c, rank=None, noise=0.05, scale=1e-3):
    k = rank or max(1, min(r, c) // 2)
    g = rng.standard_normal((r, k)) @ rng.standard_normal((k, c)) / np.sqrt(k) + noise * rng.standard_normal((r, c))
    return (scale * g).astype(np.float32)


def padded(a, dtype="f32", pad=0, fill=float("nan")):
    """The matrix on the GPU as a view of rows `pad` elements longer."""
    r, c = a.shape
    t = torch.full((r, c + pad), fill, dtype=DT[dtype], device="cuda")
    t[:, :c] = torch.from_numpy(a).cuda()
    return t[:, :c]


SETS = [
    [(1, 1)], [(1, 300), (300, 1)], [(7, 5), (5, 7), (128, 128)], [(127, 129), (129, 127)], [(128, 196), (128, 128)],
    [(256, 100), (100, 256), (20, 640)], [(300, 520)], [(520, 300), (64, 64)], [(130, 777), (777, 130)],
    [(512, 512), (1024, 128)],
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", SETS)
def test_orthogonalize(shapes, dtype):
    require_gpu()
    rng = np.random.default_rng([len(shapes), *shapes[0]])
    mats = [padded(gradient(rng, *s), dtype, pad=3 * k) for k, s in enumerate(shapes)]
    outs = [padded(np.zeros(s, np.float32), dtype, pad=5 * k) for k, s in enumerate(shapes)]
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        ref = R.orthogonalize(np_(m.float()))
        assert off(o, ref) <= bound_o(ref, dtype), (m.shape, off(o, ref) / np.linalg.norm(ref))
    opt.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cfg", [{}, dict(nesterov=0, momentum=0.0, weight_decay=0.0), dict(steps=1), dict(steps=2, momentum=0.5),
                                 dict(steps=7)])
def test_step(cfg, dtype):
    """Two updates in a row, matrices of different sizes and row strides in one call."""
    require_gpu()
    shapes = [(128, 196), (200, 72), (33, 260)]
    rng = np.random.default_rng(4)
    W = [padded(rng.standard_normal(s).astype(np.float32), pad=k) for k, s in enumerate(shapes)]
    M = [padded(gradient(rng, *s), pad=2 * k) for k, s in enumerate(shapes)]
    opt = aht.aht_muon_create(shapes, **cfg)
    refs = [(np_(w).astype(np.float64), np_(m).astype(np.float64)) for w, m in zip(W, M)]
    slack, grow = [0.0] * len(shapes), 3.4445 ** cfg.get("steps", 5) / 485
    for lr in (0.02, 0.5):
        G = [padded(gradient(rng, *s), dtype, pad=4 * k) for k, s in enumerate(shapes)]
        aht.aht_muon_step(opt, W, M, G, lr)
        aht.aht_muon_sync(opt)
        for k, s in enumerate(shapes):
            w, m, o = R.step(*refs[k], np_(G[k].float()), lr, **cfg)
            refs[k] = (w, m)
            assert off(M[k], m) <= 2 * 2e-7 * np.linalg.norm(m)
            slack[k] += 2e-7 * np.linalg.norm(w) + lr * np.sqrt(max(1, s[0] / s[1])) * (bound_o(o) * max(1, grow))
            assert off(W[k], w) <= slack[k], (s, off(W[k], w), slack[k])
    opt.close()


def test_rows_beyond_the_matrix_are_not_touched():
    require_gpu()
    rng = np.random.default_rng(0)
    W = torch.full((130, 300), 7.0, device="cuda")
    M = torch.full((130, 300), 8.0, device="cuda")
    G = padded(gradient(rng, 129, 200))
    W[:129, :200] = 0
    M[:129, :200] = 0
    opt = aht.aht_muon_create([(129, 200)])
    aht.aht_muon_step(opt, [W[:129, :200]], [M[:129, :200]], [G], 0.1)
    aht.aht_muon_sync(opt)
    assert W[:129, :200].abs().max() > 0
    for t, v in ((W, 7.0), (M, 8.0)):
        assert (t[129] == v).all() and (t[:, 200:] == v).all()


def test_low_rank_and_tiny_and_large_gradients():
    """Rank 1 and 3 of 256, and scales of 1e-12 and 1e12: the norm is taken out first."""
    require_gpu()
    rng = np.random.default_rng(1)
    shapes = [(256, 256)] * 4
    mats = [gradient(rng, 256, 256, rank=1, noise=0), gradient(rng, 256, 256, rank=3, noise=0),
            gradient(rng, 256, 256, scale=1e-12), gradient(rng, 256, 256, scale=1e12)]
    opt = aht.aht_muon_create(shapes, eps=1e-30)
    outs = [torch.empty(256, 256, device="cuda") for _ in mats]
    aht.aht_muon_orthogonalize(opt, [padded(m) for m in mats], outs)
    aht.aht_muon_sync(opt)
    for m, o in zip(mats, outs):
        ref = R.orthogonalize(m, eps=1e-30)
        assert off(o, ref) <= bound_o(ref)


def test_a_single_entry_and_identity():
    """All weight in one entry (the largest entry X can hold) and equal singular values."""
    require_gpu()
    one = np.zeros((200, 300), np.float32)
    one[150, 250] = -3.0
    eye = np.eye(200, 300, dtype=np.float32)
    opt = aht.aht_muon_create([(200, 300)] * 2)
    outs = [torch.empty(200, 300, device="cuda") for _ in range(2)]
    aht.aht_muon_orthogonalize(opt, [padded(one), padded(eye)], outs)
    aht.aht_muon_sync(opt)
    for m, o in ((one, outs[0]), (eye, outs[1])):
        ref = R.orthogonalize(m)
        assert off(o, ref) <= bound_o(ref)


def test_zero_and_not_finite_gradients():
    """Zero: no update but the decay.  NaN and inf stay within their own matrix."""
    require_gpu()
    rng = np.random.default_rng(2)
    shapes = [(100, 140)] * 4
    g = [np.zeros(shapes[0], np.float32)] + [gradient(rng, *s) for s in shapes[1:]]
    g[1][50, 60] = np.nan
    g[2][3, 4] = np.inf
    W0 = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    W, M, G = [padded(w) for w in W0], [torch.zeros(s, device="cuda") for s in shapes], [padded(v) for v in g]
    opt = aht.aht_muon_create(shapes)
    aht.aht_muon_step(opt, W, M, G, 0.1)
    aht.aht_muon_sync(opt)
    assert np.allclose(np_(W[0]), W0[0] * (1 - 0.1 * 0.01), rtol=1e-6, atol=0)
    assert W[1].isnan().all() and W[2].isnan().any()
    w, m, o = R.step(W0[3], np.zeros(shapes[3]), g[3], 0.1)
    assert off(W[3], w) <= 2e-7 * np.linalg.norm(w) + 0.1 * bound_o(o)


def test_in_place_repeatable_and_on_another_stream():
    require_gpu()
    rng = np.random.default_rng(3)
    shapes = [(300, 200), (128, 640)]
    mats = [padded(gradient(rng, *s)) for s in shapes]
    opt = aht.aht_muon_create(shapes)
    outs = [torch.empty(s, device="cuda") for s in shapes]
    aht.aht_muon_orthogonalize(opt, mats, outs)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = aht.aht_muon_create(shapes, stream=s)
    again = [m.clone() for m in mats]
    torch.cuda.synchronize()
    aht.aht_muon_orthogonalize(other, again, again)
    aht.aht_muon_sync(other)
    for a, b in zip(outs, again):
        assert torch.equal(a, b)


def test_graph_capture():
    require_gpu()
    rng = np.random.default_rng(5)
    shapes = [(128, 196), (300, 130)]
    s = torch.cuda.Stream()
    opt = aht.aht_muon_create(shapes, stream=s)
    mats, outs = [padded(gradient(rng, *v)) for v in shapes], [torch.empty(v, device="cuda") for v in shapes]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        aht.aht_muon_orthogonalize(opt, mats, outs)
    aht.aht_muon_sync(opt)
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        aht.aht_muon_orthogonalize(opt, mats, outs)
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_refusals():
    require_gpu()
    opt = aht.aht_muon_create([(8, 16)])
    w, m, g = (torch.zeros(8, 16, device="cuda") for _ in range(3))
    with pytest.raises(TypeError):
        aht.aht_muon_step(opt, [w], [m], [g.half()], 0.1)
    with pytest.raises(TypeError):
        aht.aht_muon_step(opt, [w.bfloat16()], [m], [g], 0.1)
    with pytest.raises(TypeError):
        aht.aht_muon_step(opt, [w.cpu()], [m], [g], 0.1)
    with pytest.raises(ValueError):
        aht.aht_muon_step(opt, [w, w], [m], [g], 0.1)
    with pytest.raises(ValueError):
        aht.aht_muon_step(opt, [w], [m[:, :8]], [g], 0.1)
    with pytest.raises(ValueError):                                  # column-major
        aht.aht_muon_step(opt, [torch.zeros(16, 8, device="cuda").t()], [m], [g], 0.1)
    with pytest.raises(ValueError):                                  # rows that overlap
        aht.aht_muon_step(opt, [torch.zeros(16, device="cuda").expand(8, 16)], [m], [g], 0.1)
    with pytest.raises(aht.AhtError):
        aht.aht_muon_step(opt, [w], [m], [g], float("nan"))
    with pytest.raises(TypeError):
        aht.aht_muon_orthogonalize(opt, [g], [g.bfloat16()])
    assert not w.any()


def test_an_expired_allocation_leaves_nothing():
    """Sizes are refused before anything is allocated."""
    require_gpu()
    free = torch.cuda.mem_get_info()[0]
    for shapes, cfg in (([(0, 4)], {}), ([(4, 16385)], {}), ([(4, 4)] * 49, {}), ([(4, 4)], dict(momentum=1.0)),
                        ([(4, 4)], dict(steps=0)), ([(4, 4)], dict(eps=0.0)), ([(4, 4)], dict(weight_decay=-1.0))):
        with pytest.raises(aht.AhtError):
            aht.aht_muon_create(shapes, **cfg)
    assert torch.cuda.mem_get_info()[0] == free
