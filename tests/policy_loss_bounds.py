"""How far the fp32 policy loss may be from the 64-bit reference, entry by entry.

With e = 2^-24, p the row's softmax, xm = x - max x, ym = y - max y, Ex = sum p |xm|, Ey = sum p |ym|:
- A sum over the row goes through n additions: a thread's own, one after the other (A / 32 of a row of up to 8192
  actions, which a warp may have, A / 256 beyond, A up to 64), and those that join 32 lanes and 16 warps.  An exponential is off
  by 2^-22 of itself (2 ulp) and 2 e |xm| from its argument; moving a sum to a new maximum is one more factor of that kind,
  16 of them at most for rows in random order.  Sums of one sign are therefore off, relative to themselves, by
      d = (n + 64 + 4 (Ex + Ey)) 2^-24 + 2^-22,   with 16 2^-22 = 64 2^-24.
- logp is off by  l = d + 2^-22 (1 + |log s| + |xm_action|); log s, u / s, t / s and log sy give H and KL within
      c = d (3 + 2 Ex + 2 Ey) + 2^-22 (1 + Ex + Ey + |log s| + |log sy|) + l.
- With at the weight of the action's own term (of slope dat in logp), an entry w p_j (k0 + k1 xm_j - k2 ym_j) is formed
  from terms of together at most
      B_j = |at| + (ent + kl) (|xm_j| + log s + H) + kl (|ym_j| + |log sy| + |KL|)
  and is off by  w p_j (B_j (2 d + 2^-20 + 2 e |xm_j|) + 2 (ent + kl) c + 2 dat l), the action's own by
  w (2^-21 |at| + 2 dat l) more, each entry by half a step of its type, and by w B_j 2^-126 where its exponential is below
  the normal numbers.
All of it is proportional to p_j: a gradient of 0 in the place of any entry of weight is out of the bounds."""
import numpy as np


def _sum_rows(x, ok):
    x = np.where(ok, x, -np.inf)
    top = x.max(1, keepdims=True)
    xm = x - top
    return xm, np.log(np.exp(xm).sum(1))


@np.errstate(invalid="ignore", over="ignore")     # (of masked places, which nothing below reads)
def bounds(x, actions, old_logp, adv, legal=None, weight=None, ref_logits=None, ref_logp=None, clip_low=0.2, clip_high=0.2,
           kl_coef=0.0, ent_coef=0.0, half_step=2.0 ** -24, want=None):
    """want: the reference's (stats, logp, dlogits).  -> tolerances of the three.  Rows take part with finite sums."""
    M, A = x.shape
    stats, logp, grad = want
    rows = np.arange(M)
    a = np.clip(actions.astype(np.int64), 0, A - 1)
    ok = np.ones((M, A), bool) if legal is None else legal != 0
    part = (actions >= 0) & (actions < A) & ok[rows, a] & (np.where(ok, x, -np.inf) > -np.inf).any(1)
    ok = np.where(part[:, None], ok, True)
    x = np.where(part[:, None], x, 0.0)
    w = np.full(M, 1.0 / M) if weight is None else weight.astype(np.float64)
    w = np.where(part, w, 0.0)
    xm, ls = _sum_rows(x, ok)
    p = np.exp(xm - ls[:, None])
    live = ok & (xm > -np.inf)
    ax = np.abs(np.where(live & (xm > -1e4), xm, 0.0))    # (beyond, the exponential is 0 in either arithmetic)
    Ex = (p * ax).sum(1)
    H = -(p * np.where(live, xm - ls[:, None], 0.0)).sum(1)
    ay, Ey, lsy, KL, kl = np.zeros((M, A)), np.zeros(M), np.zeros(M), np.zeros(M), kl_coef
    if ref_logits is not None:
        ym, lsy = _sum_rows(np.where(part[:, None], ref_logits, 0.0), ok)
        ay = np.abs(np.where(live & (ym > -1e4), ym, 0.0))
        Ey = (p * ay).sum(1)
        KL = (p * np.where(live & (ym > -np.inf), (xm - ls[:, None]) - (ym - lsy[:, None]), 0.0)).sum(1)
    else:
        kl = 0.0
    n = A if A <= 64 else A / 32 + 6 if A <= 8192 else A / 256 + 24
    e = 2.0 ** -24
    d = (n + 64 + 4 * (Ex + Ey)) * e + 2.0 ** -22
    xa = np.where(live[rows, a], ax[rows, a], 0.0)
    lp = np.where(part & (logp > -np.inf), logp, 0.0)
    lt = d + 2.0 ** -22 * (1 + np.abs(ls) + xa)
    c = d * (3 + 2 * Ex + 2 * Ey) + 2.0 ** -22 * (1 + Ex + Ey + np.abs(ls) + np.abs(lsy)) + lt
    ratio = np.exp(np.minimum(np.where(part, logp - old_logp, 0.0), 80))
    at, dat = np.abs(adv) * ratio, np.abs(adv) * ratio
    if ref_logp is not None:
        far = np.exp(np.minimum(np.where(part, ref_logp - lp, 0.0), 80))
        at, dat = at + kl_coef * np.abs(far - 1), dat + kl_coef * far
        KL = far - 1 - np.where(part, ref_logp - lp, 0.0)
    B = at[:, None] + (ent_coef + kl) * (ax + ls[:, None] + H[:, None]) + kl * (ay + np.abs(lsy)[:, None] + np.abs(KL)[:, None])
    c2 = 2 * (ent_coef + kl) * c + 2 * dat * lt
    tol = w[:, None] * (p * (B * (2 * d[:, None] + 2.0 ** -20 + 2 * e * ax) + c2[:, None]) + B * 2.0 ** -126)
    tol[rows, a] += w * (2.0 ** -21 * at + 2 * dat * lt)
    tol = np.where(ok & part[:, None], tol + half_step * (np.abs(grad) + tol), 0.0)
    # l, the clipped term, KL, H, 1 where clipped, 1: a row's value with its error, summed
    own = np.stack([at + kl_coef * np.abs(KL) + ent_coef * H, at, np.abs(KL), H, np.ones(M), np.ones(M)], 1) * 2.0 ** -22
    kl_off = 2 * c if ref_logits is not None else 0 * c if ref_logp is None else 2 * lt * np.abs(far - 1) + 2 * lt * lt
    off = np.stack([2 * dat * lt + kl_coef * kl_off + 2 * ent_coef * c, 2 * dat * lt, kl_off, 2 * c, 0 * c, 0 * c], 1)
    return (w[:, None] * (own + off)).sum(0) + 2.0 ** -23 * np.abs(stats), np.where(part, lt, 0.0), tol
