"""Muon step in fp64 (the definition; test infrastructure only): momentum, quintic Newton-Schulz steps (Jordan et al. 2024), the weights' step."""
import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def orthogonalize(u, steps, trace=None):
    """u [rows, cols] -> X; `trace` (a list) gets every step's X in front of it, shorter side first."""
    norm = np.sqrt((u * u).sum())
    x = u / norm if norm > 0 else u * 0
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(steps):
        if trace is not None:
            trace.append(x)
        a = x @ x.T
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.T if tall else x


def step(w, grad, m, lr, momentum, nesterov, weight_decay, steps, scale):
    """Returns the new weights, the new momentum, the orthogonal update and the update before it."""
    m = momentum * m + grad
    u = grad + momentum * m if nesterov else m
    x = orthogonalize(u, steps)
    return (1 - lr * weight_decay) * w - lr * scale * x, m, x, u


def steepest(s):
    """The largest factor by which one step enlarges a small change of X (in the Frobenius norm) where X has the singular values s: the derivative of the
    polynomial and its divided differences, of values with equal and with opposite signs."""
    s = np.concatenate([s, -s])
    p = A * s + B * s ** 3 + C * s ** 5
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.abs((p[:, None] - p[None]) / (s[:, None] - s[None]))
    return max(np.nanmax(np.where(np.isfinite(q), q, 0.0)), np.abs(A + 3 * B * s ** 2 + 5 * C * s ** 4).max(), A)
