"""Root-mean-square norm of the rows of x + residual and its gradients in fp64 (the definition; test infrastructure only)."""
import numpy as np


def forward(x, residual=None, weight=None, eps=1e-5):
    """x [rows, cols].  Returns y, x + residual, rstd."""
    z = x if residual is None else x + residual
    r = 1 / np.sqrt((z * z).mean(1) + eps)
    y = z * r[:, None]
    return y if weight is None else y * weight, z, r


def backward(dy, total, weight, rstd, dtotal=None):
    """Returns dx, dweight, from the rows' own rstd."""
    h = total * rstd[:, None]
    k = dy if weight is None else dy * weight
    dx = rstd[:, None] * (k - h * (k * h).mean(1, keepdims=True))
    return dx if dtotal is None else dx + dtotal, (dy * h).sum(0)
