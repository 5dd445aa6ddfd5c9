"""The bounds of policy_loss_bounds.py hold for plain fp32 arithmetic and tell wrong results from right ones (no GPU)."""
import numpy as np
import pytest

import policy_loss_ref as R
from policy_loss_bounds import bounds

COEF = dict(clip_low=0.2, clip_high=0.25, kl_coef=0.05, ent_coef=0.01)


def data(M, A, seed):
    g = np.random.default_rng(seed)
    x = (2 * g.standard_normal((M, A))).astype(np.float32).astype(np.float64)
    y = (x + 0.3 * g.standard_normal((M, A))).astype(np.float32).astype(np.float64)
    a = g.integers(0, A, M)
    lp = x - np.log(np.exp(x).sum(1, keepdims=True))
    old = (lp[np.arange(M), a] + 0.1 * g.standard_normal(M)).astype(np.float32).astype(np.float64)
    return dict(x=x, actions=a, old_logp=old, adv=g.standard_normal(M), ref_logits=y)


def plain32(d, leave_out=None):
    """The loss in fp32, sums in numpy's order; ``leave_out``: a slice of every row that the sums miss."""
    f = np.float32
    x, y = d["x"].astype(f), d["ref_logits"].astype(f)
    M, A = x.shape
    w, rows = f(1 / M), np.arange(M)
    xm, ym = x - x.max(1, keepdims=True), y - y.max(1, keepdims=True)
    ex, ey = np.exp(xm), np.exp(ym)
    in_sum = np.ones(A, f)
    if leave_out is not None:
        in_sum[leave_out] = 0
    s, sy = (ex * in_sum).sum(1, dtype=f), (ey * in_sum).sum(1, dtype=f)
    lp, lq = xm - np.log(s)[:, None], ym - np.log(sy)[:, None]
    p = ex / s[:, None]
    H, KL = -(p * lp * in_sum).sum(1, dtype=f), (p * (lp - lq) * in_sum).sum(1, dtype=f)
    logp, adv = lp[rows, d["actions"]], d["adv"].astype(f)
    ratio = np.exp(logp - d["old_logp"].astype(f))
    clipped = ((adv > 0) & (ratio > f(1.25))) | ((adv < 0) & (ratio < f(0.8)))
    pg = -np.minimum(ratio * adv, np.clip(ratio, f(0.8), f(1.25)) * adv)
    at = np.where(clipped, f(0), -adv * ratio)
    g = p * (f(0.01) * (lp + H[:, None]) + f(0.05) * (lp - lq - KL[:, None]) - at[:, None])
    g[rows, d["actions"]] += at
    pg, KL_, H_, c = (float((w * v.astype(np.float64)).sum()) for v in (pg, KL, H, clipped))
    return np.array([pg + 0.05 * KL_ - 0.01 * H_, pg, KL_, H_, c, 1.0]), logp.astype(np.float64), (w * g).astype(np.float64)


@pytest.mark.parametrize("M,A", [(40, 6), (40, 64), (40, 127), (30, 1000), (6, 8200), (3, 65536)])
def test_bounds_hold_and_tell(M, A):
    d = data(M, A, A)
    want = R.loss(**d, **COEF)
    tol = bounds(**d, **COEF, want=want)
    for have, ref, t in zip(plain32(d), want, tol):
        assert (np.abs(have - ref) <= t).all(), float((np.abs(have - ref) - t).max())
    stats, logp, grad = tol
    # a gradient of zeros, of any entry of weight; a KL of 0; a row's logp off by a ten-thousandth
    assert (np.abs(want[2]) > grad).mean() > 0.98
    assert (np.abs(want[2]) > 20 * grad).mean() > 0.9
    assert np.abs(want[0][2]) > 20 * stats[2] and np.abs(want[0][3]) > 1000 * stats[3]
    assert (logp < 1e-4).all()
    # a vector of eight that the sums miss
    if A >= 64:
        wrong = plain32(d, slice(A // 2, A // 2 + 8))
        assert (np.abs(wrong[1] - want[1]) > logp).any() and (np.abs(wrong[2] - want[2]) > grad).any()
