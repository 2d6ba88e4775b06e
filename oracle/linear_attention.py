"""Linear attention with a decay for each head, step by step in fp64.

    S_t = l keep_{t-1} S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   l = exp(log_decay[h])

keep_t = 0 where dones[t, n] is set; s_last = keep S behind the last step that exists.  Shapes: q, k [T, N, H, Dk], v [T, N, H, Dv],
s0 [N, H, Dk, Dv].  What is dropped is dropped by selection, so values that are not finite stay where they belong.
"""
import numpy as np


def _setup(q, v, s0, dones, lengths):
    T, N, H, Dk = q.shape
    Dv = v.shape[-1]
    S = np.zeros((N, H, Dk, Dv)) if s0 is None else np.array(s0, np.float64)
    ends = np.zeros((T, N), bool) if dones is None else np.asarray(dones).reshape(T, N) != 0
    length = np.full(N, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return T, N, H, Dk, Dv, S, ends, length


def _outer(a, b):
    return a[..., :, None] * b[..., None, :]


def _pick(mask, a, b):
    return np.where(mask.reshape(mask.shape + (1,) * (a.ndim - 1)), a, b)


def _decay(log_decay):
    return np.exp(np.asarray(log_decay, np.float64))[None, :, None, None]


def forward(q, k, v, log_decay, scale, s0=None, dones=None, lengths=None):
    """Returns o [T, N, H, Dv] and s_last."""
    with np.errstate(invalid="ignore", over="ignore"):
        q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
        T, N, H, Dk, Dv, S, ends, length = _setup(q, v, s0, dones, lengths)
        l, o = _decay(log_decay), np.zeros((T, N, H, Dv))
        for t in range(T):
            here = t < length
            new = l * S + _outer(k[t], v[t])
            o[t] = _pick(here, scale * (q[t][..., :, None] * new).sum(2), np.zeros_like(o[t]))
            S = _pick(here, _pick(ends[t], np.zeros_like(S), new), S)
    return o, S


def backward(q, k, v, log_decay, scale, do, ds_last=None, s0=None, dones=None, lengths=None):
    """Returns dq, dk, dv, ds0."""
    with np.errstate(invalid="ignore", over="ignore"):
        q, k, v, do = (np.asarray(x, np.float64) for x in (q, k, v, do))
        T, N, H, Dk, Dv, S, ends, length = _setup(q, v, s0, dones, lengths)
        l = _decay(log_decay)
        dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
        for t in range(T):
            here = t < length
            new = l * S + _outer(k[t], v[t])
            dq[t] = _pick(here, scale * (new * do[t][..., None, :]).sum(3), dq[t])
            S = _pick(here, _pick(ends[t], np.zeros_like(S), new), S)
        Z = np.zeros((N, H, Dk, Dv)) if ds_last is None else np.array(ds_last, np.float64)     # behind step t, towards the state kept there
        for t in range(T - 1, -1, -1):
            here = t < length
            dS = _pick(ends[t], np.zeros_like(Z), Z) + scale * _outer(q[t], do[t])
            dk[t] = _pick(here, (dS * v[t][..., None, :]).sum(3), dk[t])
            dv[t] = _pick(here, (dS * k[t][..., :, None]).sum(2), dv[t])
            Z = _pick(here, l * dS, Z)
    return dq, dk, dv, Z


def step(q, k, v, log_decay, scale, s_in=None, reset=None):
    """One step: q, k [N, H, Dk], v [N, H, Dv].  Returns o, s_out."""
    reset = None if reset is None else np.asarray(reset) != 0
    s0 = s_in
    if s0 is not None and reset is not None:
        s0 = _pick(reset, np.zeros_like(s0), np.asarray(s0, np.float64))
    o, S = forward(q[None], k[None], v[None], log_decay, scale, s0)
    return o[0], S


def magnitudes(fn, *args, **kw):
    """The same sums over absolute values: what rounding errors are relative to."""
    a = [np.abs(np.asarray(x, np.float64)) if isinstance(x, np.ndarray) and x.ndim == 4 else x for x in args]
    kw = {n: (np.abs(np.asarray(x, np.float64)) if isinstance(x, np.ndarray) and x.ndim == 4 else x) for n, x in kw.items()}
    return fn(*a, **kw)
