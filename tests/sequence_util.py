"""Inputs and error bounds of the sequence operators' tests.

Bounds are derived, not fitted.  With u = 2^-24 (half a step of fp32) every term of a sum passes through a number of fp32 roundings, each
worth at most u of the term, so a result is off by at most (roundings) u (sum of the terms' absolute values); the oracles run over
absolute values give that sum.  The result's own rounding to its type adds eps / 2 of it (and half the type's smallest number).
"""
import numpy as np
import torch

from oracle import linear_attention as ola

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def rounding(dtype, ref):
    """What rounding to the type costs: half a step of the value, half the smallest step."""
    f = torch.finfo(dtype)
    return 1.01 * f.eps / 2 * np.abs(ref) + f.tiny * f.eps / 2


def attention_roundings(T, Dk, Dv):
    """A score is a sum of D products, weighted (4 roundings: two factors of at most two units each), summed over at most 16 positions; a
    state takes 4 + 16 roundings a chunk of 16 positions that it lives through (at most T / 16 + 1 of them), and pieces that are
    walked apart are joined in 2 each (at least 64 positions long); reading it sums D products.  Generously, and for any chunking of
    at most 2 roundings a position:"""
    return 2 * max(Dk, Dv) + 2 * T + 64


def held(ref):
    """fp64 values as fp32 holds them: a state of 1e-88 is zero there."""
    return ref.astype(np.float32).astype(np.float64)


def check(name, got, ref, bound):
    """|got - ref| <= bound element by element."""
    got = got.detach().float().cpu().numpy().astype(np.float64) if isinstance(got, torch.Tensor) else np.asarray(got, np.float64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    if ref.size == 0:
        return
    bound = np.broadcast_to(bound, ref.shape)
    off = np.abs(got - ref)
    worse = ~(off <= bound)
    if worse.any():
        i = np.unravel_index(int(np.argmax(np.where(np.isnan(off), np.inf, off / np.maximum(bound, 1e-300)))), off.shape)
        raise AssertionError("%s%s: %.9g, not %.9g (off by %.3g, at most %.3g; %d of %d out)" % (name, list(i), got[i], ref[i], off[i], bound[i],
                                                                                           int(worse.sum()), off.size))


def typed(x, dtype):
    """fp64 numpy -> CPU tensor of the type; the oracle is fed what it holds."""
    return torch.as_tensor(np.asarray(x)).to(dtype)


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Attention:
    """Inputs of one call on the CPU, their oracle results, and copies on the GPU (strided as asked)."""

    def __init__(self, seed, T, N, H, Dk, Dv, dtype="fp32", done_p=0.0, s0=True, ragged=False, layout="dense", decays=None):
        g = np.random.default_rng(seed)
        self.T, self.N, self.H, self.Dk, self.Dv, self.dtype, self.layout = T, N, H, Dk, Dv, TYPES[dtype], layout
        r = lambda *s: g.normal(size=s)  # noqa: E731
        self.q, self.k = typed(r(T, N, H, Dk), self.dtype), typed(r(T, N, H, Dk), self.dtype)
        self.v, self.do = typed(r(T, N, H, Dv), self.dtype), typed(r(T, N, H, Dv), self.dtype)
        if layout == "shared_key":
            self.k = self.k[:, :, :1].expand(T, N, H, Dk)
        self.s0 = typed(r(N, H, Dk, Dv), torch.float32) if s0 else None
        self.ds_last = typed(r(N, H, Dk, Dv), torch.float32) if s0 else None
        # the fastest forgets in two steps, the slowest hardly at all
        self.log_decay = typed(-np.exp(np.linspace(np.log(0.7), np.log(1e-4), H)) if decays is None else np.array(decays), torch.float32)
        self.dones = torch.as_tensor((g.random((T, N)) < done_p).astype(np.uint8)) if done_p else None
        self.lengths = torch.as_tensor(g.integers(0, T + 1, N).astype(np.int32)) if ragged else None
        if ragged and N > 1:
            self.lengths[0], self.lengths[1] = T, 0
        self.scale = float(np.float32(1 / np.sqrt(Dk)))
        self.roundings = attention_roundings(T, Dk, Dv)

    def args(self):
        return (f64(self.q), f64(self.k), f64(self.v), f64(self.log_decay), self.scale)

    def kw(self):
        return dict(s0=f64(self.s0), dones=None if self.dones is None else self.dones.numpy(),
                    lengths=None if self.lengths is None else self.lengths.numpy())

    def place(self, x):
        """x on the GPU, its rows laid out as the case asks."""
        T, N, H, D = x.shape
        if self.layout == "dense":
            return x.contiguous().cuda()
        if self.layout == "shared_key":
            return x[:, :, :1].contiguous().cuda().expand(T, N, H, D) if x.stride(2) == 0 and H > 1 else x.contiguous().cuda()
        if self.layout == "batch_first":                       # [N, T, H, D]
            return x.permute(1, 0, 2, 3).contiguous().cuda().permute(1, 0, 2, 3)
        if self.layout == "head_first":                        # [N, H, T, D]
            return x.permute(1, 2, 0, 3).contiguous().cuda().permute(2, 0, 1, 3)
        assert self.layout == "odd"                            # rows one value further apart, starting one value in
        wide = torch.full((T, N, H, D + 1), float("nan"), dtype=x.dtype, device="cuda")
        wide[..., 1:] = x.cuda()
        return wide[..., 1:]

    def empty(self, D):
        return self.place(torch.full((self.T, self.N, self.H, D), float("nan"), dtype=self.dtype))

    def on_gpu(self, rx):
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.g = dict(q=self.place(self.q), k=self.place(self.k), v=self.place(self.v), do=self.place(self.do), s0=dev(self.s0), ds_last=dev(self.ds_last))
        self.la = rx.LinearAttn(self.dtype, self.T, self.N, self.H, self.Dk, self.Dv, dev(self.log_decay), self.scale, dev(self.dones), dev(self.lengths))
        return self.g, self.la

    def state(self):
        return torch.full((self.N, self.H, self.Dk, self.Dv), float("nan"), device="cuda")

    def run_forward(self, rx):
        g, la = self.on_gpu(rx)
        o, s = self.empty(self.Dv), self.state()
        rx.rslx_linear_attention(la, g["q"], g["k"], g["v"], g["s0"], o, s, rx.workspace(rx.rslx_linear_attention_workspace_bytes(la)))
        return o, s

    def run_backward(self, rx):
        g, la = self.on_gpu(rx)
        dq, dk, dv, ds0 = self.empty(self.Dk), self.empty(self.Dk), self.empty(self.Dv), self.state()
        rx.rslx_linear_attention_backward(la, g["q"], g["k"], g["v"], g["s0"], g["do"], g["ds_last"], dq, dk, dv, ds0,
                                          rx.workspace(rx.rslx_linear_attention_backward_workspace_bytes(la)))
        return dq, dk, dv, ds0

    def check_forward(self, o, s):
        ro, rs = ola.forward(*self.args(), **self.kw())
        mo, ms = ola.magnitudes(ola.forward, *self.args(), **self.kw())
        check("o", o, ro, rounding(self.dtype, ro) + self.roundings * U * mo)
        check("s_last", s, held(rs), self.roundings * U * ms)

    def check_backward(self, dq, dk, dv, ds0):
        more = dict(self.kw(), do=f64(self.do), ds_last=f64(self.ds_last))
        ref = ola.backward(*self.args(), **more)
        mag = ola.magnitudes(ola.backward, *self.args(), **more)
        for name, got, r, m in zip(("dq", "dk", "dv"), (dq, dk, dv), ref, mag):
            check(name, got, r, rounding(self.dtype, r) + self.roundings * U * m)
        check("ds0", ds0, held(ref[3]), self.roundings * U * mag[3])
