"""Gated linear recurrence per sequence n and channel d, step by step in fp64 (the definition; test infrastructure only).

    f = sigmoid(g),  h_t = f_t k_{t-1} h_{t-1} + (1 - f_t) x_t,   h_{-1} = s0
k_t = 0 behind a step that ends an episode (dones), k_{-1} = 1; the state behind the sequence is k_{T-1} h_{T-1}.  With lengths, steps at and
behind lengths[n] do not exist: outputs there are zero and the state stays as it is.
"""
import numpy as np


def gates(g):
    """sigmoid(g) and 1 - sigmoid(g)."""
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def _there(t, lengths):
    return (t < np.clip(lengths, 0, None))[:, None] if lengths is not None else True


def forward(x, g, s0=None, dones=None, lengths=None):
    """x, g [T, N, D]; s0 [N, D].  Returns h [T, N, D], the last state, and the states that every step starts from."""
    T, N, D = x.shape
    f, rest = gates(g)
    s = np.zeros((N, D)) if s0 is None else np.array(s0, np.float64)
    h, entered = np.zeros((T, N, D)), np.zeros((T, N, D))
    for t in range(T):
        here = _there(t, lengths)
        entered[t] = s
        with np.errstate(invalid="ignore"):
            new = f[t] * s + rest[t] * x[t]
        h[t] = np.where(here, new, 0.0)
        if dones is not None:
            new = np.where(dones[t].astype(bool)[:, None], 0.0, new)
        s = np.where(here, new, s)
    return h, s, entered


def backward(x, g, dh, ds_last=None, s0=None, dones=None, lengths=None):
    """Returns dx, dg, ds0."""
    T, N, D = x.shape
    f, rest = gates(g)
    entered = forward(x, g, s0, dones, lengths)[2]
    d = np.zeros((N, D)) if ds_last is None else np.array(ds_last, np.float64)
    dx, dg = np.zeros((T, N, D)), np.zeros((T, N, D))
    for t in range(T - 1, -1, -1):
        here = _there(t, lengths)
        kept = d if dones is None else np.where(dones[t].astype(bool)[:, None], 0.0, d)
        now = kept + dh[t]
        with np.errstate(invalid="ignore"):
            dx[t] = np.where(here, rest[t] * now, 0.0)
            dg[t] = np.where(here, f[t] * rest[t] * now * (entered[t] - x[t]), 0.0)
            d = np.where(here, f[t] * now, d)
    return dx, dg, d


def sizes(x, g, s0=None, dones=None, lengths=None, each=1.0):
    """Sums of the absolute values of every state's terms [T, N, D], and the errors that gather in the states where every step adds `each` of that sum:
    e_t = f k e_{t-1} + each m_t, likewise."""
    m, _, _ = forward(np.abs(x), g, None if s0 is None else np.abs(s0), dones, lengths)
    _, rest = gates(g)
    with np.errstate(divide="ignore", invalid="ignore"):
        e, last, _ = forward(np.where(rest > 0, each * m / rest, 0.0), g, None, dones, lengths)
    return m, e, last
