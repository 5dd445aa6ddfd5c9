"""The gated linear recurrence on the GPU (aht_glr_forward, aht_glr_backward) against the
formulas in 64 bits (tests/glr_ref.py), on the rounded inputs.

Tolerances, fixed before the first run.  Every fp32 gate is a few operations of 2^-24
relative error each (about 10, so 1e-6); a state sums terms whose weights decay, and the
slowest test channel keeps a = 0.999, so errors of a (6e-8 each) accumulate over at most
about 1000 steps of like-signed terms: 6e-5 of the state, at one channel; relative to the
whole array's norm far less.  fp32 outputs: 2e-5 in the 2-norm, and elementwise 4e-4 of
max(rms, |value|).  bf16 outputs round once, to 8 significant bits: at most 2^-8 = 3.9e-3 of
an element, so 4e-3 elementwise and, as every element may be that far off (an array of one
is), in the 2-norm.  dlam and the states are fp32 whatever the type."""
import numpy as np
import pytest
import torch

from paper_2609_13716_gb300 import aht

import glr_ref as R
from gpu_util import np_, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def near(got, ref, dtype="f32", what=""):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    if not ref.size:
        return
    rms = np.sqrt(np.mean(ref ** 2))
    if rms == 0:
        assert not got.any(), what
        return
    rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    worst = np.max(np.abs(got - ref) / np.maximum(rms, np.abs(ref)))
    lim = (2e-5, 4e-4) if dtype == "f32" else (4e-3, 4e-3)
    assert rel <= lim[0] and worst <= lim[1], f"{what}: rel {rel:.3g}, worst {worst:.3g}"


def sequence(rng, T, N, D, dtype, layout, scale=1.0, count=1):
    """count [T][N][D] tensors; layout: time-major, env-major, or slices of a wider row."""
    v = (rng.standard_normal((count, T, N, D)) * scale).astype(np.float32)
    out = []
    if layout == "fused":
        whole = torch.full((T, N, count * D + 3), float("nan"), dtype=DT[dtype], device="cuda")
        for k in range(count):
            whole[:, :, k * D:(k + 1) * D] = torch.from_numpy(v[k]).cuda()
            out.append(whole[:, :, k * D:(k + 1) * D])
    elif layout == "env":
        out = [torch.from_numpy(np.ascontiguousarray(u.swapaxes(0, 1))).cuda().to(DT[dtype]).transpose(0, 1) for u in v]
    else:
        out = [torch.from_numpy(u).cuda().to(DT[dtype]) for u in v]
    return out


def problem(T, N, D, dtype, layout="time", resets=0.05, ragged=False, seed=0):
    rng = np.random.default_rng([seed, T, N, D])
    x, r, i = sequence(rng, T, N, D, dtype, layout, 1.2, 3)
    decay = rng.uniform(0.9, 0.999, D)
    p = dict(x=x, r=r, i=i, lam=torch.from_numpy(np.log(np.expm1(-np.log(decay) / 8)).astype(np.float32)).cuda(),
             h0=torch.from_numpy(rng.standard_normal((N, D)).astype(np.float32)).cuda(), reset=None, lengths=None)
    if resets:
        p["reset"] = torch.from_numpy((rng.random((T, N)) < resets).astype(np.uint8)).cuda()
    if ragged:
        lens = rng.integers(0, T + 1, N)
        lens[0] = 0
        lens[-1] = T
        p["lengths"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    p["dh"], = sequence(rng, T, N, D, dtype, layout)
    p["dh_last"] = torch.from_numpy(rng.standard_normal((N, D)).astype(np.float32)).cuda()
    return p


def host(p):
    return {k: None if v is None else np_(v.float() if v.dtype == torch.bfloat16 else v) for k, v in p.items()}


def fwd(p, h="like", ckpt=True, h_last=None, h0="h0", **kw):
    T, N, D = p["x"].shape
    h = torch.full_like(p["x"], float("nan")) if isinstance(h, str) else h
    h_last = torch.full((N, D), float("nan"), device="cuda") if h_last is None else h_last
    ck = torch.full(aht.aht_glr_ckpt_shape(T, N, D), float("nan"), device="cuda") if ckpt else None
    aht.aht_glr_forward(p["x"], p["r"], p["i"], p["lam"], h, reset=p["reset"], lengths=p["lengths"],
                        h0=p["h0"] if h0 == "h0" else h0, h_last=h_last, ckpt=ck, **kw)
    return h, h_last, ck


def bwd(p, ckpt, dh="dh", dh_last="dh_last", **kw):
    T, N, D = p["x"].shape
    out = {k: torch.full_like(p["x"], float("nan")) for k in ("dx", "dr", "di")}
    out["dlam"], out["dh0"] = (torch.full(s, float("nan"), device="cuda") for s in ((D,), (N, D)))
    ws = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device="cuda")
    aht.aht_glr_backward(p["x"], p["r"], p["i"], p["lam"], ckpt, p["dh"] if dh == "dh" else dh, out["dx"], out["dr"],
                         out["di"], out["dlam"], ws, reset=p["reset"], lengths=p["lengths"],
                         dh_last=p["dh_last"] if dh_last == "dh_last" else dh_last, dh0=out["dh0"], **kw)
    return out


def check_all(p, dtype):
    h, h_last, ck = fwd(p)
    got = bwd(p, ck)
    q = host(p)
    rh, rl, before = R.forward(q["x"], q["r"], q["i"], q["lam"], q["reset"], q["lengths"], q["h0"])
    near(np_(h.float()), rh, dtype, "h")
    near(np_(h_last), rl, "f32", "h_last")
    ref = dict(zip(("dx", "dr", "di", "dlam", "dh0"), R.backward(q["x"], q["r"], q["i"], q["lam"], before, q["dh"],
                                                                 q["reset"], q["lengths"], q["dh_last"])))
    for k, v in ref.items():
        near(np_(got[k].float()), v, dtype if k in ("dx", "dr", "di") else "f32", k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,layout,ragged", [
    (1, 1, 1, "time", False), (1, 5, 128, "time", False), (2, 3, 7, "env", False), (7, 4, 64, "fused", True),
    (8, 2, 33, "time", True), (9, 3, 128, "env", True), (63, 2, 130, "time", False), (64, 5, 96, "fused", False),
    (65, 1, 256, "time", False), (129, 7, 20, "env", True), (515, 2, 200, "fused", False), (1030, 1, 66, "time", False),
    (300, 40, 64, "time", True),
])
def test_forward_and_backward(T, N, D, layout, ragged, dtype):
    require_gpu()
    check_all(problem(T, N, D, dtype, layout, ragged=ragged), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_stream(dtype):
    """One stream long enough to be split over many thread groups, few resets."""
    require_gpu()
    check_all(problem(5003, 1, 64, dtype, resets=0.002), dtype)


def test_no_reset_no_lengths_no_initial_state():
    require_gpu()
    p = problem(50, 3, 40, "f32", resets=0)
    h, last, _ = fwd(p, h0=None)
    q = host(p)
    rh, rl, _ = R.forward(q["x"], q["r"], q["i"], q["lam"])
    near(np_(h), rh, what="h")
    near(np_(last), rl, what="h_last")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_in_a_row_equal_the_sequence(dtype):
    """T = 1 calls that carry the state in place give the sequence's h and final state."""
    require_gpu()
    T, N, D = 37, 19, 128
    p = problem(T, N, D, dtype)
    h, last, _ = fwd(p)
    state = p["h0"].clone()
    one = torch.empty(T, N, D, dtype=DT[dtype], device="cuda")
    for t in range(T):
        aht.aht_glr_forward(p["x"][t:t + 1], p["r"][t:t + 1], p["i"][t:t + 1], p["lam"], one[t:t + 1],
                            reset=p["reset"][t:t + 1].contiguous(), h0=state, h_last=state)
    near(np_(one.float()), np_(h.float()), dtype, "h")
    near(np_(state), np_(last), "f32", "state")


def test_split_call_continues_the_sequence():
    require_gpu()
    p = problem(100, 3, 48, "f32")
    _, last, _ = fwd(p)
    state = p["h0"].clone()
    for lo, hi in ((0, 33), (33, 34), (34, 100)):
        aht.aht_glr_forward(p["x"][lo:hi], p["r"][lo:hi], p["i"][lo:hi], p["lam"], reset=p["reset"][lo:hi].contiguous(),
                            h0=state, h_last=state)
    near(np_(state), np_(last), what="state")


@pytest.mark.parametrize("T", [40, 700])
def test_masked_steps_may_hold_anything(T):
    """NaN and inf past an env's length reach no output; h and the gradients are 0 there."""
    require_gpu()
    p = problem(T, 6, 64, "f32", ragged=True)
    clean = {k: v.clone() for k, v in p.items()}
    dead = torch.arange(T, device="cuda")[:, None] >= p["lengths"]
    for k, bad in (("x", float("nan")), ("r", float("inf")), ("i", float("-inf")), ("dh", float("nan"))):
        p[k] = torch.where(dead[..., None], torch.full_like(p[k], bad), p[k])
    h0, l0, c0 = fwd(clean)
    h1, l1, c1 = fwd(p)
    assert torch.equal(h0, h1) and torch.equal(l0, l1) and not h1[dead].any()
    assert torch.equal(l1[p["lengths"] == 0], p["h0"][p["lengths"] == 0])   # no step at all: the state stays
    a, b = bwd(clean, c0), bwd(p, c1)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    for k in ("dx", "dr", "di"):
        assert not b[k][dead].any()


@pytest.mark.parametrize("T", [40, 700])
def test_reset_drops_a_state_that_is_not_finite(T):
    """NaN or inf in one episode stays in it, forward and backward."""
    require_gpu()
    p = problem(T, 4, 64, "f32", resets=0)
    p["reset"] = torch.zeros(T, 4, dtype=torch.uint8, device="cuda")
    cut = T // 2 + 1
    p["reset"][cut] = 1
    clean_h, clean_last, ck = fwd(p)
    clean = bwd(p, ck)
    p["x"][cut - 1, 0] = float("nan")
    p["h0"][1] = float("inf")
    h, last, ck = fwd(p)
    assert torch.equal(h[cut:], clean_h[cut:]) and torch.equal(last, clean_last)
    assert h[cut - 1, 0].isnan().all() and h[0, 1].isinf().all()
    got = bwd(p, ck)
    for k in ("dx", "dr", "di"):
        assert torch.equal(got[k][cut:], clean[k][cut:]), k
    p["dh"][cut + 1, 2] = float("nan")      # a gradient of the second episode
    got = bwd(p, ck)
    assert torch.equal(got["dx"][:cut, 2], clean["dx"][:cut, 2]) and got["dx"][cut, 2].isnan().all()


def test_saturated_gates():
    """Gates at 0 and 1 and extreme decay parameters: finite, and the formulas' limits."""
    require_gpu()
    vals = [-200.0, -90.0, -30.0, -3.0, 0.0, 3.0, 30.0, 90.0, 200.0]
    T, D = 24, len(vals) ** 2
    p = problem(T, 2, D, "f32", resets=0.1)
    grid = torch.tensor([[a, b] for a in vals for b in vals], device="cuda")
    p["r"] = grid[:, 0].expand(T, 2, D).contiguous()
    p["i"] = grid[:, 1].expand(T, 2, D).contiguous()
    p["lam"] = torch.tensor([-60.0, -20.0, -5.0, 0.0, 5.0, 40.0], device="cuda").repeat(D)[:D].contiguous()
    check_all(p, "f32")


def test_gradient_against_differences():
    """Directional derivatives of a scalar loss by central differences of the forward pass
    (fp32 h in, differences summed in fp64; step 2^-7 keeps both errors below 1e-3)."""
    require_gpu()
    T, N, D = 23, 3, 16
    p = problem(T, N, D, "f32", resets=0.1)
    _, _, ck = fwd(p)
    got = bwd(p, ck)
    rng = np.random.default_rng(3)

    def loss(q):
        h, last, _ = fwd(q, ckpt=False)
        return float((h.double() * q["dh"].double()).sum() + (last.double() * q["dh_last"].double()).sum())

    for name, grad in (("x", "dx"), ("r", "dr"), ("i", "di"), ("lam", "dlam"), ("h0", "dh0")):
        v = torch.from_numpy(rng.standard_normal(tuple(p[name].shape)).astype(np.float32)).cuda()
        eps = 2.0 ** -7
        up, dn = dict(p), dict(p)
        up[name], dn[name] = p[name] + eps * v, p[name] - eps * v
        num = (loss(up) - loss(dn)) / (2 * eps)
        ana = float((got[grad].double() * v.double()).sum())
        scale = float((got[grad].double().norm() * v.double().norm()))
        assert abs(num - ana) <= 2e-3 * max(abs(ana), 0.1 * scale), (name, num, ana)


def test_broadcast_inputs_and_missing_outer_gradients():
    """Inputs may repeat rows (stride 0); dh alone, dh_last alone, and no lam or h0 gradient."""
    require_gpu()
    T, N, D = 30, 4, 32
    p = problem(T, N, D, "f32")
    p["i"] = p["i"][:1, :1].expand(T, N, D)
    q = host(p)
    h, last, ck = fwd(p, h=torch.empty(T, N, D, device="cuda"))
    rh, rl, before = R.forward(q["x"], q["r"], q["i"], q["lam"], q["reset"], q["lengths"], q["h0"])
    near(np_(h), rh, what="h")
    dx, dr, di = (torch.full((T, N, D), float("nan"), device="cuda") for _ in range(3))
    for dh, dl in ((p["dh"], None), (None, p["dh_last"])):
        aht.aht_glr_backward(p["x"], p["r"], p["i"], p["lam"], ck, dh, dx, dr, di, reset=p["reset"], dh_last=dl)
        ref = R.backward(q["x"], q["r"], q["i"], q["lam"], before, None if dh is None else q["dh"], q["reset"], None,
                         None if dl is None else q["dh_last"])
        for got, want, k in ((dx, ref[0], "dx"), (dr, ref[1], "dr"), (di, ref[2], "di")):
            near(np_(got), want, what=k)


def test_unaligned_views():
    """Rows that begin at any element: views offset by one element, odd strides."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        T, N, D = 70, 3, 64
        p = problem(T, N, D, dtype)
        for k in ("x", "r", "i", "dh"):
            wide = torch.zeros(T, N, D + 5, dtype=DT[dtype], device="cuda")
            wide[:, :, 1:1 + D] = p[k]
            p[k] = wide[:, :, 1:1 + D]
        check_all(p, dtype)


def test_empty_sequence():
    require_gpu()
    p = problem(0, 3, 8, "f32", resets=0)
    last = torch.full((3, 8), float("nan"), device="cuda")
    aht.aht_glr_forward(p["x"], p["r"], p["i"], p["lam"], None, h0=p["h0"], h_last=last)
    assert torch.equal(last, p["h0"])
    got = bwd(p, torch.empty(0, 3, 8, device="cuda"))
    assert torch.equal(got["dh0"], p["dh_last"]) and not got["dlam"].any()


def test_calls_repeat_bit_for_bit_and_run_on_another_stream():
    require_gpu()
    p = problem(400, 9, 96, "bf16", ragged=True)
    h, last, ck = fwd(p)
    g = bwd(p, ck)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    h2, last2, ck2 = fwd(p, stream=s)
    g2 = bwd(p, ck2, stream=s)
    s.synchronize()
    assert torch.equal(h, h2) and torch.equal(last, last2) and torch.equal(ck, ck2)
    for k in g:
        assert torch.equal(g[k], g2[k]), k


def test_graph_capture():
    require_gpu()
    T, N, D = 64, 8, 64
    p = problem(T, N, D, "f32")
    want, wl, ck = fwd(p)
    ref = bwd(p, ck)
    out = {k: torch.empty_like(p["x"]) for k in ("h", "dx", "dr", "di")}
    last, dlam, dh0 = torch.empty(N, D, device="cuda"), torch.empty(D, device="cuda"), torch.empty(N, D, device="cuda")
    ws = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        aht.aht_glr_forward(p["x"], p["r"], p["i"], p["lam"], out["h"], reset=p["reset"], h0=p["h0"], h_last=last, ckpt=ck)
        aht.aht_glr_backward(p["x"], p["r"], p["i"], p["lam"], ck, p["dh"], out["dx"], out["dr"], out["di"], dlam, ws,
                             reset=p["reset"], dh_last=p["dh_last"], dh0=dh0)
    for _ in range(2):
        ck.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["h"], want) and torch.equal(last, wl)
        for k in ("dx", "dr", "di"):
            assert torch.equal(out[k], ref[k])
        assert torch.equal(dlam, ref["dlam"]) and torch.equal(dh0, ref["dh0"])


def test_refusals():
    require_gpu()
    p = problem(8, 2, 16, "f32")
    h = torch.empty_like(p["x"])
    args = (p["x"], p["r"], p["i"], p["lam"])
    with pytest.raises(TypeError):
        aht.aht_glr_forward(p["x"].half(), p["r"], p["i"], p["lam"], h)
    with pytest.raises(TypeError):
        aht.aht_glr_forward(p["x"], p["r"].bfloat16(), p["i"], p["lam"], h)
    with pytest.raises(TypeError):
        aht.aht_glr_forward(*args, h.cpu())
    with pytest.raises(ValueError):
        aht.aht_glr_forward(p["x"], p["r"][:, :1], p["i"], p["lam"], h)
    with pytest.raises(ValueError):                                 # channels not contiguous
        aht.aht_glr_forward(p["x"], p["r"], p["i"], p["lam"], torch.empty(8, 16, 2, device="cuda").transpose(1, 2))
    with pytest.raises(ValueError):                                 # written rows that share memory
        aht.aht_glr_forward(*args, torch.empty(1, 2, 16, device="cuda").expand(8, 2, 16))
    with pytest.raises(ValueError):
        aht.aht_glr_forward(*args, h, lengths=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(aht.AhtError):                               # no output at all
        aht.aht_glr_forward(*args, None)
    g = [torch.empty_like(p["x"]) for _ in range(3)]
    ck = torch.empty(1, 2, 16, device="cuda")
    with pytest.raises(aht.AhtError):
        aht.aht_glr_backward(*args, None, p["dh"], *g)              # no checkpoints
    with pytest.raises(aht.AhtError):
        aht.aht_glr_backward(*args, ck, p["dh"], g[0], None, g[2])
    with pytest.raises(aht.AhtError):                               # dlam without its workspace
        aht.aht_glr_backward(*args, ck, p["dh"], *g, dlam=torch.empty(16, device="cuda"))
    with pytest.raises(ValueError):
        aht.aht_glr_backward(*args, torch.empty(2, 2, 16, device="cuda"), p["dh"], *g)
