"""Rows masked by the logits themselves, and rows whose legal logits are all very low, against the 64-bit reference
(tolerances: policy_loss_bounds.py)."""
import numpy as np
import pytest
import torch

import policy_loss_ref as R
import test_gpu_policy_loss as L
from policy_loss_bounds import bounds

pytestmark = pytest.mark.gpu
INF = float("inf")


def check(d):
    got = L.run(d)
    a = {k: L.to64(v) for k, v in dict(x=d["logits"], actions=d["actions"], old_logp=d["old_logp"], adv=d["advantages"], legal=d["legal"],
                                       weight=d["weight"], ref_logits=d["ref_logits"], ref_logp=d["ref_logp"]).items()}
    with np.errstate(invalid="ignore", over="ignore"):
        want = R.loss(**a, **L.COEF)
        tol = bounds(**a, **L.COEF, want=want, half_step=2.0 ** -8 if d["logits"].dtype is torch.bfloat16 else 2.0 ** -24)
    for n, ref, t in zip(("stats", "logp", "dlogits"), want, tol):
        have = L.to64(got[n])
        bad = ~(np.abs(have - ref) <= t)
        assert not bad.any(), (n, int(bad.sum()), np.argwhere(bad)[:4].tolist(), have[bad][:4], ref[bad][:4], t[bad][:4])
    return got


def masked(M, A, dtype, spans, value, ref="logits", seed=0, both=False):
    """Logits of ``value`` over spans of columns, another span for each row; actions elsewhere."""
    d = L.make(M, A, dtype, ref, seed=seed, actions=torch.int64)
    torch.manual_seed(0)
    d["actions"] = torch.randint(0, A, (M,), device="cuda")
    x = d["logits"].clone()
    y = d["ref_logits"].clone() if ref == "logits" else None
    for m in range(M):
        lo, hi = spans[m % len(spans)]
        x[m, lo:hi] = value
        if both:
            y[m, lo:hi] = value
        left = [j for j in range(A) if not lo <= j < hi]
        d["actions"][m] = left[(7 * m + seed) % len(left)]
    lp = torch.log_softmax(x.double(), 1).gather(1, d["actions"][:, None])[:, 0]
    d["old_logp"] = (lp + 0.1).float()
    d["logits"], d["ref_logits"] = x, y
    if ref == "logp":
        d["ref_logp"] = (lp + 0.2).float()
    return d


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("ref", ["logits", "logp", "none"])
@pytest.mark.parametrize("A", [48, 65, 100, 128, 256, 1500, 9001])
def test_whole_vectors_of_no_probability(A, ref, dtype):
    """-inf over the head of a row, its middle, its tail, most of it, and single vectors; the reference is finite there
    and counts."""
    spans = [(0, 8), (0, A // 4), (A // 3, A // 3 + 16), (A - 8, A), (A // 2, A), (4, A - 3), (0, A - 1), (1, A), (0, 0)]
    check(masked(18, A, dtype, spans, -INF, ref, seed=A))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("value", [-INF, "lowest", -1.5e30, -1e30, -1e9])
@pytest.mark.parametrize("A", [100, 1500, 9001])
def test_other_values_that_leave_no_probability(A, value, dtype):
    v = torch.finfo(dtype).min if value == "lowest" else value
    check(masked(12, A, dtype, [(0, 8), (0, A // 2), (A // 2, A), (3, A - 2)], v, seed=1))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("A", [48, 100, 256, 1500, 9001])
def test_masked_in_the_reference_as_well(A, dtype):
    """The reference's probability is 0 where the policy's is: nothing of KL."""
    d = masked(12, A, dtype, [(0, 8), (0, A // 2), (A // 2, A), (3, A - 2)], -INF, seed=2, both=True)
    with np.errstate(invalid="ignore"):
        check(d)


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("with_mask", [False, True])
@pytest.mark.parametrize("level", [-1e29, -1.3e30, -2e30, -1e35, -1e38])
@pytest.mark.parametrize("A", [48, 100, 256, 1500, 9001])
def test_rows_of_very_low_logits(A, level, with_mask, dtype):
    """Every legal logit lies far below any other row's, at a level and twice it; what is not legal is 0 or above, and the
    reference's as low.  The probabilities are those of the logits at the level, 1 / their number."""
    M = 6
    d = L.make(M, A, dtype, "logits", seed=3, actions=torch.int64)
    torch.manual_seed(0)
    x, y = torch.full((M, A), 2 * level, device="cuda"), torch.full((M, A), 2 * level, device="cuda")
    top = torch.rand(M, A, device="cuda") < 0.4
    d["actions"] = torch.randint(0, A, (M,), device="cuda")
    top[torch.arange(M), d["actions"]] = True
    x[top], y[top] = level, level
    d["legal"] = None
    if with_mask:
        d["legal"] = (torch.rand(M, A, device="cuda") < 0.5).to(torch.uint8)
        d["legal"][:, :min(32, A // 2)] = 0
        d["legal"][torch.arange(M), d["actions"]] = 1
        x[d["legal"] == 0], y[d["legal"] == 0] = 1.0, 3.0
    d["logits"], d["ref_logits"] = x.to(dtype), y.to(dtype)
    live = top if d["legal"] is None else top & (d["legal"] != 0)
    d["old_logp"] = -live.sum(1).float().log() + 0.1
    check(d)


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("A", [100, 256, 1500, 9001])
def test_contiguous_ranges_that_are_not_legal(A, dtype):
    d = L.make(16, A, dtype, "logits", legal=True, seed=4, actions=torch.int64)
    torch.manual_seed(0)
    d["legal"][:] = 0
    d["actions"] = torch.randint(0, A, (16,), device="cuda")
    for m in range(16):
        lo = (m * A // 16) % A
        d["legal"][m, lo:lo + max(1, A // 5)] = 1
    d["legal"][torch.arange(16), d["actions"]] = 1
    x = d["logits"].double().masked_fill(d["legal"] == 0, -INF)
    d["old_logp"] = (torch.log_softmax(x, 1).gather(1, d["actions"][:, None])[:, 0] + 0.1).float()
    check(d)
