"""The gated linear recurrence and its gradient in 64 bits, one step at a time (numpy),
written from the formulas in include/aht.h."""
import numpy as np


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def forward(x, r, i, lam, reset=None, lengths=None, h0=None):
    """x, r, i [T][N][D] -> h [T][N][D], h_last [N][D], the states before each step."""
    T, N, D = x.shape
    s = 8 * softplus(lam.astype(np.float64))
    y = np.zeros((N, D)) if h0 is None else h0.astype(np.float64).copy()
    h, before = np.zeros((T, N, D)), np.zeros((T, N, D))
    for t in range(T):
        before[t] = y
        for n in range(N):
            if lengths is not None and t >= lengths[n]:
                continue
            q = s * _sigmoid(r[t, n].astype(np.float64))
            b = np.sqrt(-np.expm1(-2 * q)) * _sigmoid(i[t, n].astype(np.float64)) * x[t, n]
            y[n] = b if reset is not None and reset[t, n] else np.exp(-q) * y[n] + b
            h[t, n] = y[n]
    return h, y, before


def backward(x, r, i, lam, before, dh=None, reset=None, lengths=None, dh_last=None):
    """-> dx, dr, di [T][N][D], dlam [D], dh0 [N][D]."""
    T, N, D = x.shape
    lam = lam.astype(np.float64)
    s = 8 * softplus(lam)
    dx, dr, di = (np.zeros((T, N, D)) for _ in range(3))
    ds = np.zeros(D)
    p = np.zeros((N, D)) if dh_last is None else dh_last.astype(np.float64).copy()
    for t in reversed(range(T)):
        for n in range(N):
            if lengths is not None and t >= lengths[n]:
                continue
            xx, rho, iota = x[t, n].astype(np.float64), _sigmoid(r[t, n].astype(np.float64)), _sigmoid(i[t, n].astype(np.float64))
            q = s * rho
            a, beta = np.exp(-q), np.sqrt(-np.expm1(-2 * q))
            rs = reset is not None and bool(reset[t, n])
            g = p[n] + (0 if dh is None else dh[t, n].astype(np.float64))
            dx[t, n] = g * beta * iota
            di[t, n] = g * beta * xx * iota * (1 - iota)
            # dL/dq through a = exp(-q) and beta = sqrt(1 - a^2), d beta / dq = a^2 / beta;
            # times q stays finite as q -> 0
            qb = np.where(beta > 0, q / np.where(beta > 0, beta, 1), 0)
            qdq = -q * a * g * (0 if rs else before[t, n]) + qb * a * a * g * iota * xx
            dr[t, n] = qdq * (1 - rho)
            ds += np.where(s > 0, qdq / np.where(s > 0, s, 1), 0)
            p[n] = 0 if rs else a * g
    return dx, dr, di, 8 * ds * _sigmoid(lam), p
