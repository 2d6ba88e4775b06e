"""Layer norm over the rows of a matrix in fp64: y = (x - m) r w + b, m the mean, r = 1 / sqrt(variance + eps)."""
import numpy as np


def forward(x, weight=None, bias=None, eps=1e-5):
    """Returns y, mean, rstd."""
    x = np.asarray(x, np.float64)
    m = x.mean(1)
    r = 1.0 / np.sqrt(((x - m[:, None]) ** 2).mean(1) + eps)
    y = (x - m[:, None]) * r[:, None]
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, m, r


def backward(dy, x, weight, mean, rstd):
    """Returns dx, dweight, dbias for the given statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    m, r = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    h = (x - m) * r
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = r * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)
