"""Cases of the sequence-model training operators: the gated linear recurrence over a
collected trajectory (forward, one serving step, and forward + backward), the
Newton-Schulz orthogonalisation of a matrix update, and the optimiser step that applies it.

``run`` computes an operator in its plain form (elementary torch operations in 32 bits,
rounded once at the end), or, where ``own`` is true, through the framework's entry points.
``exact`` computes the same outputs from the definitions in 64 bits, one step at a time.
"""
import math

import torch

own = False

C_GATE = 8.0                            # exponent of the recurrence gate
NS = (3.4445, -4.7750, 2.0315)          # quintic of the orthogonalisation
NS_STEPS = 5
LR, MOMENTUM, DECAY, EPS = 0.02, 0.95, 0.01, 1e-7

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _glr(name, op, T, N, D, dtype, layout="time", lengths=False, episode=50):
    c = dict(op=op, T=T, N=N, D=D, dtype=dtype, layout=layout, lengths=lengths, episode=episode)
    return dict(c, name=name) if name else c


def _muon(name, op, shapes, dtype):
    c = dict(op=op, shapes=shapes, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: one step of 64 live envs (the 64-env LBF configuration), latency only
        _glr("step 64x128 bf16", "scan", 1, 64, 128, "bf16"),
        # the value/feature pass over the PPO collection: 16384 envs x 128 steps, model size 128
        _glr("scan 128x16384x128 bf16", "scan", 128, 16384, 128, "bf16"),
        # one packed stream of many episodes, gates sliced from one fused projection
        _glr("scan 65537x1x896 f32 fused", "scan", 65537, 1, 896, "f32", layout="fused"),
        # evaluation episodes of different lengths (400-step kitchen), env-major tensors
        _glr("scan 400x509x200 f32 ragged", "scan", 400, 509, 200, "f32", layout="env", lengths=True),
        # training pass over a 4096-env collection
        _glr("train 128x4096x128 bf16", "train", 128, 4096, 128, "bf16"),
        # few long streams, wide state
        _glr("train 4096x8x512 f32", "train", 4096, 8, 512, "f32", layout="fused", episode=400),
        # a handful of short games (97 turns), odd sizes, some of them empty
        _glr("train 97x33x100 bf16 ragged", "train", 97, 33, 100, "bf16", layout="env", lengths=True),
        # the MLP learner's hidden matrices
        _muon("update mlp", "update", "128x196,128x128", "f32"),
        # the recurrent actor-critic's matrices: encoder and two heads of 1024 units
        _muon("update heads", "update", "128x196,128x128,1024x128*2,1024x1024*4", "f32"),
        # one large matrix, bf16 gradient
        _muon("update 2048x4096 bf16", "update", "2048x4096", "bf16"),
        # a tall and a wide odd matrix
        _muon("orthogonalise odd bf16", "ortho", "777x130,130x777*2", "bf16"),
        # a square one on its own
        _muon("orthogonalise 1024 f32", "ortho", "1024x1024", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "train", "train", "update", "ortho"])
    if op in ("scan", "train"):
        most = 2.0e8 if op == "scan" else 6.0e7
        while True:
            T = 1 if op == "scan" and rng.random() < 0.25 else _log_int(rng, 2, 65537)
            N, D = _log_int(rng, 1, 16384), _log_int(rng, 16, 1000)
            if rng.random() < 0.6:
                D = max(16, D // 8 * 8)
            if 2000 <= T * N * D <= most:
                break
        return _glr(None, op, T, N, D, rng.choice(["f32", "bf16"]), rng.choice(["time", "fused", "env"]),
                    rng.random() < 0.35, rng.choice([20, 50, 97, 400]))
    parts, budget = [], 1.1e11
    for _ in range(rng.randint(1, 3)):
        r, c = _log_int(rng, 16, 2048), _log_int(rng, 16, 2900)
        k = rng.randint(1, 4)
        m, n = min(r, c), max(r, c)
        cost = k * (3.0 * m * m * n + m ** 3)
        if cost > budget and parts:
            continue
        k = max(1, min(k, int(budget / (cost / k))))
        budget -= cost
        parts.append("%dx%d*%d" % (r, c, k))
    return _muon(None, op, ",".join(parts), rng.choice(["f32", "bf16"]))


def _shapes(text):
    out = []
    for p in text.split(","):
        s, _, k = p.partition("*")
        r, c = (int(v) for v in s.split("x"))
        out += [(r, c)] * int(k or 1)
    return out


def work(case):
    if case["op"] in ("scan", "train"):
        T, N, D = case["T"], case["N"], case["D"]
        e = 4 if case["dtype"] == "f32" else 2
        small = 8 * N * D + T * N + 4 * D
        if case["op"] == "scan":        # x, r, i read, h written
            return {"bytes": 4 * e * T * N * D + small, "flops": 20.0 * T * N * D}
        # and x, r, i, dh read, dx, dr, di written
        return {"bytes": 11 * e * T * N * D + 3 * small, "flops": 60.0 * T * N * D}
    e = 4 if case["dtype"] == "f32" else 2
    b = f = 0.0
    for r, c in _shapes(case["shapes"]):
        m, n = min(r, c), max(r, c)
        f += NS_STEPS * (3.0 * m * m * n + m ** 3)      # X X^T and A A symmetric, B X full
        b += r * c * (16 + e if case["op"] == "update" else 2 * e)
    return {"bytes": b, "flops": f}


# ---- inputs -----------------------------------------------------------------------------
def _seq(g, case, count, scale):
    """`count` [T][N][D] sequences of the case's layout."""
    T, N, D, dt = case["T"], case["N"], case["D"], DTYPES[case["dtype"]]
    rnd = lambda *s: (torch.randn(*s, device="cuda", generator=g) * scale).to(dt)  # noqa: E731
    if case["layout"] == "fused":       # slices of one projection's output
        return list(rnd(T, N, count * D).split(D, dim=2))
    if case["layout"] == "env":         # env-major storage
        return [rnd(N, T, D).transpose(0, 1) for _ in range(count)]
    return [rnd(T, N, D) for _ in range(count)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=case)
    if case["op"] in ("scan", "train"):
        T, N, D, dt = case["T"], case["N"], case["D"], DTYPES[case["dtype"]]
        s["x"], s["r"], s["i"] = _seq(g, case, 3, 1.2)
        a = 0.9 + 0.099 * torch.rand(D, device="cuda", generator=g)      # slow modes
        s["lam"] = torch.log(torch.expm1(-torch.log(a) / C_GATE))
        s["reset"] = (torch.rand(T, N, device="cuda", generator=g) < 1.0 / case["episode"]).to(torch.uint8)
        s["lengths"] = torch.randint(0, T + 1, (N,), device="cuda", generator=g, dtype=torch.int32) if case["lengths"] else None
        s["h0"] = 0.5 * torch.randn(N, D, device="cuda", generator=g)
        if case["op"] == "train":
            s["dh"] = _seq(g, case, 1, 1.0)[0]
            s["dh_last"] = torch.randn(N, D, device="cuda", generator=g)
        if own:                         # the buffers a training loop keeps
            from paper_2609_13716_gb300 import aht
            like = lambda t: torch.empty_strided(t.shape, t.stride(), dtype=dt, device="cuda")  # noqa: E731
            dense = torch.empty(T, N, D, dtype=dt, device="cuda") if case["layout"] != "env" else like(s["x"])
            s["h"], s["h_last"] = dense, torch.empty(N, D, device="cuda")
            if case["op"] == "train":
                s["ckpt"] = torch.empty(aht.aht_glr_ckpt_shape(T, N, D), device="cuda")
                s["dx"], s["dr"], s["di"] = (torch.empty_like(dense) for _ in range(3))
                s["dlam"], s["dh0"] = torch.empty(D, device="cuda"), torch.empty(N, D, device="cuda")
                s["ws"] = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device="cuda")
        return s
    dt = DTYPES[case["dtype"]]
    s["shapes"] = _shapes(case["shapes"])
    s["G"], s["M"], s["W"] = [], [], []

    def gradient(r, c):                 # a decaying spectrum of sample directions plus noise
        k = max(1, min(r, c) // 4)
        u = torch.randn(r, k, device="cuda", generator=g) * torch.exp(-4.0 * torch.arange(k, device="cuda") / k)
        return 1e-3 * (u @ torch.randn(k, c, device="cuda", generator=g) / math.sqrt(k)
                       + 0.05 * torch.randn(r, c, device="cuda", generator=g))

    for r, c in s["shapes"]:
        s["G"].append(gradient(r, c).to(dt))
        if case["op"] == "update":
            s["M"].append(10.0 * gradient(r, c))
            s["W"].append(torch.randn(r, c, device="cuda", generator=g) / math.sqrt(c))
    if own:
        from paper_2609_13716_gb300 import aht
        s["opt"] = aht.aht_muon_create(s["shapes"], momentum=MOMENTUM, weight_decay=DECAY, eps=EPS)
        s["O"] = [torch.empty_like(v) for v in s["G"]] if case["op"] == "ortho" else None
    return s


# ---- plain forms ------------------------------------------------------------------------
def _scan_plain(a, b):
    """y_t = a_t y_{t-1} + b_t over dim 0 (y_{-1} = 0), by doubling."""
    k = 1
    while k < a.shape[0]:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _gates_plain(s):
    x, r, i = (s[k].float() for k in ("x", "r", "i"))
    T, N = x.shape[:2]
    softplus = torch.log1p(torch.exp(-s["lam"].abs())) + s["lam"].clamp(min=0)
    rho, iota = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-i))
    q = C_GATE * softplus * rho
    a, beta = torch.exp(-q), torch.sqrt(-torch.expm1(-2 * q))
    keep = (s["reset"] == 0).unsqueeze(2)
    live = torch.ones(T, N, 1, dtype=torch.bool, device=x.device)
    if s["lengths"] is not None:
        live = (torch.arange(T, device=x.device).unsqueeze(1) < s["lengths"]).unsqueeze(2)
    return x, rho, iota, softplus, q, a, beta, keep, live


def _glr_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    x, rho, iota, softplus, q, a, beta, keep, live = _gates_plain(s)
    decay = torch.where(live, torch.where(keep, a, torch.zeros_like(a)), torch.ones_like(a))
    b = torch.where(live, beta * iota * x, torch.zeros_like(x))
    b = torch.cat([(b[0] + decay[0] * s["h0"]).unsqueeze(0), b[1:]])
    h = _scan_plain(decay, b)
    out = {"h": torch.where(live, h, torch.zeros_like(h)).to(dt), "h_last": h[-1].clone()}
    if case["op"] == "scan":
        return out
    dh = torch.where(live, s["dh"].float(), torch.zeros_like(h))
    dh = torch.cat([dh[:-1], (dh[-1] + s["dh_last"]).unsqueeze(0)])
    nxt = torch.cat([decay[1:], torch.ones_like(decay[:1])])
    g = _scan_plain(nxt.flip(0), dh.flip(0)).flip(0)
    prev = torch.cat([s["h0"].unsqueeze(0), h[:-1]])
    prev = torch.where(keep, prev, torch.zeros_like(prev))
    g_in = torch.where(live, g, torch.zeros_like(g))
    w = q * a * prev * g_in - (q / beta) * a * a * iota * x * g_in
    out["dx"] = (g_in * beta * iota).to(dt)
    out["di"] = (g_in * beta * x * iota * (1 - iota)).to(dt)
    out["dr"] = (-(1 - rho) * w).to(dt)
    sig = 1 / (1 + torch.exp(-s["lam"]))
    out["dlam"] = -w.sum(dim=(0, 1)) * sig / softplus
    out["dh0"] = decay[0] * g[0]
    return out


def _orthogonal_plain(u):
    x = u / (torch.sqrt((u * u).sum()) + EPS)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(NS_STEPS):
        y = x @ x.t()
        x = NS[0] * x + (NS[1] * y + NS[2] * (y @ y)) @ x
    return x.t() if tall else x


def _muon_plain(s):
    out = []
    for k, (r, c) in enumerate(s["shapes"]):
        g = s["G"][k]
        if s["case"]["op"] == "ortho":
            out.append(_orthogonal_plain(g.float()).to(g.dtype))
            continue
        s["M"][k].mul_(MOMENTUM).add_(g.float())
        o = _orthogonal_plain(g.float() + MOMENTUM * s["M"][k])
        s["W"][k].mul_(1 - LR * DECAY).sub_(LR * math.sqrt(max(1.0, r / c)) * o)
    return out if s["case"]["op"] == "ortho" else {"W": s["W"], "M": s["M"]}


# ---- the framework's entry points ---------------------------------------------------------
def _glr_own(s):
    from paper_2609_13716_gb300 import aht
    train = s["case"]["op"] == "train"
    aht.aht_glr_forward(s["x"], s["r"], s["i"], s["lam"], s["h"], reset=s["reset"], lengths=s["lengths"],
                        h0=s["h0"], h_last=s["h_last"], ckpt=s["ckpt"] if train else None)
    out = {"h": s["h"], "h_last": s["h_last"]}
    if train:
        aht.aht_glr_backward(s["x"], s["r"], s["i"], s["lam"], s["ckpt"], s["dh"], s["dx"], s["dr"], s["di"],
                             s["dlam"], s["ws"], reset=s["reset"], lengths=s["lengths"], dh_last=s["dh_last"],
                             dh0=s["dh0"])
        out.update(dx=s["dx"], dr=s["dr"], di=s["di"], dlam=s["dlam"], dh0=s["dh0"])
    return out


def _muon_own(s):
    from paper_2609_13716_gb300 import aht
    if s["case"]["op"] == "ortho":
        aht.aht_muon_orthogonalize(s["opt"], s["G"], s["O"])
        return s["O"]
    aht.aht_muon_step(s["opt"], s["W"], s["M"], s["G"], LR)
    return {"W": s["W"], "M": s["M"]}


def run(state):
    glr = state["case"]["op"] in ("scan", "train")
    if own:
        return _glr_own(state) if glr else _muon_own(state)
    return _glr_plain(state) if glr else _muon_plain(state)


# ---- 64 bits ------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("scan", "train"):
        return _glr_exact(case, s)
    out, W, M = [], [], []
    for k, (r, c) in enumerate(s["shapes"]):
        g = s["G"][k].double().cpu()
        if case["op"] == "update":
            m = MOMENTUM * s["M"][k].double().cpu() + g
            M.append(m)
            u = g + MOMENTUM * m
        else:
            u = g
        u = u / (u.norm() + EPS)
        # the polynomial of the singular values, through the Gram matrix of the short side
        left = r <= c
        for _ in range(NS_STEPS):
            gram = u @ u.t() if left else u.t() @ u
            poly = NS[1] * gram + NS[2] * gram @ gram
            u = NS[0] * u + (poly @ u if left else u @ poly)
        out.append(u)
        if case["op"] == "update":
            W.append((1 - LR * DECAY) * s["W"][k].double().cpu() - LR * math.sqrt(max(1.0, r / c)) * u)
    return out if case["op"] == "ortho" else {"W": W, "M": M}


def _glr_exact(case, s):
    T, N, D = case["T"], case["N"], case["D"]
    f64 = torch.float64
    lam = s["lam"].to(f64)
    soft = torch.nn.functional.softplus(lam, threshold=100.0)
    reset, lens = s["reset"].bool(), s["lengths"]
    live_all = torch.ones(T, N, dtype=torch.bool, device="cuda") if lens is None else torch.arange(T, device="cuda")[:, None] < lens
    step = max(1, 30_000_000 // (N * D))          # steps whose gates are formed at once

    def gates(t0):
        t1 = min(T, t0 + step)
        x = s["x"][t0:t1].to(f64)
        rho, iota = torch.sigmoid(s["r"][t0:t1].to(f64)), torch.sigmoid(s["i"][t0:t1].to(f64))
        q = C_GATE * soft * rho
        a, beta = torch.exp(-q), torch.sqrt(-torch.expm1(-2 * q))
        live, keep = live_all[t0:t1, :, None], ~reset[t0:t1, :, None]
        return x, rho, iota, q, a, beta, live, keep

    state = s["h0"].to(f64)
    h, before = torch.empty(T, N, D, dtype=f64, device="cuda"), []
    for t0 in range(0, T, step):
        x, rho, iota, q, a, beta, live, keep = gates(t0)
        before.append(state)
        decay = torch.where(live, a * keep, torch.ones_like(a))
        b = torch.where(live, beta * iota * x, torch.zeros_like(a))
        y = torch.empty_like(b)
        for t in range(b.shape[0]):
            state = torch.addcmul(b[t], decay[t], state, out=y[t])
        state = state.clone()
        h[t0:t0 + step] = torch.where(live, y, torch.zeros_like(y))
    out = {"h": h, "h_last": state}
    if case["op"] == "scan":
        return out
    carry = s["dh_last"].to(f64)                  # gradient of the state after step t
    dx, dr, di = (torch.empty(T, N, D, dtype=f64, device="cuda") for _ in range(3))
    dlam = torch.zeros(D, dtype=f64, device="cuda")
    for k in reversed(range(len(before))):
        t0 = k * step
        x, rho, iota, q, a, beta, live, keep = gates(t0)
        decay = torch.where(live, a * keep, torch.ones_like(a))
        b = torch.where(live, beta * iota * x, torch.zeros_like(a))
        n = b.shape[0]
        prev, st = torch.empty_like(b), before[k]
        for t in range(n):
            prev[t] = st
            st = b[t] + decay[t] * st
        dh = torch.where(live, s["dh"][t0:t0 + n].to(f64), torch.zeros_like(b))
        g = torch.empty_like(b)
        for t in reversed(range(n)):
            torch.add(dh[t], carry, out=g[t])
            carry = decay[t] * g[t]
        g = torch.where(live, g, torch.zeros_like(g))
        dbeta = g * iota * x
        da = g * prev * keep - dbeta * a / beta
        dq = -a * da                              # dL/dq
        dx[t0:t0 + n] = g * beta * iota
        di[t0:t0 + n] = g * beta * x * iota * (1 - iota)
        dr[t0:t0 + n] = dq * q * (1 - rho)
        dlam += (dq * rho).sum(dim=(0, 1)) * C_GATE * torch.sigmoid(lam)
    out.update(dx=dx, dr=dr, di=di, dlam=dlam, dh0=carry)
    return out
