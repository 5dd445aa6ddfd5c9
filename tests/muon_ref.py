"""The orthogonalised update in 64 bits (numpy), written from the formulas in include/aht.h."""
import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def orthogonalize(u, eps=1e-7, steps=5):
    x = u.astype(np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        g = x.T @ x if x.shape[0] > x.shape[1] else x @ x.T
        p = A * np.eye(g.shape[0]) + B * g + C * (g @ g)
        x = x @ p if x.shape[0] > x.shape[1] else p @ x
    return x


def step(W, M, G, lr, momentum=0.95, weight_decay=0.01, eps=1e-7, nesterov=1, steps=5):
    """-> W, M, and the orthogonal factor."""
    M = momentum * M.astype(np.float64) + G
    o = orthogonalize(G + momentum * M if nesterov else M, eps, steps)
    return (1 - lr * weight_decay) * W.astype(np.float64) - lr * np.sqrt(max(1.0, W.shape[0] / W.shape[1])) * o, M, o
