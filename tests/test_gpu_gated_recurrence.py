"""Gated linear recurrence on the GPU against fp64.

Bounds: a gate passes at most 6 roundings of u = 2^-24 (exp's two, 1 + e, the reciprocal's two, a product), a step of the recurrence two more, and a
join of two pieces as many as a step; so every step adds at most 12 u of the sum of its terms' absolute values to a state's error, which the gates behind it
carry on.  Gates of 16 bits take the exponential of a rounded product, |g| u more: 12 u for gates up to 12 as here.  The recurrence over these errors gives the bound (oracle.gated_recurrence.sizes).  Gates and products below fp32's smallest normal number,
2^-126, may be zero: a step loses at most 2^-126 (1 + |x|) of a state to that.
"""
import numpy as np
import pytest
import torch

from oracle import gated_recurrence as ogr
from sequence_util import TYPES, U, check, f64, rounding, typed

pytestmark = pytest.mark.gpu

STEPS = {torch.float32: 12 * U, torch.bfloat16: 24 * U, torch.float16: 24 * U}


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


class Case:
    """Inputs of one call on the CPU, and copies on the GPU, laid out as asked."""

    def __init__(self, seed, T, N, D, dtype="fp32", done_p=0.0, s0=True, ragged=False, layout="side"):
        g = np.random.default_rng(seed)
        self.T, self.N, self.D, self.dtype, self.layout = T, N, D, TYPES[dtype], layout
        self.step = STEPS[self.dtype]
        self.x, self.dh = (typed(g.normal(size=(T, N, D)), self.dtype) for _ in range(2))
        self.g = typed(np.clip(g.normal(size=(T, N, D)) * 1.5 + np.linspace(-2, 6, D), -12, 12), self.dtype)
        self.s0, self.ds_last = ((typed(g.normal(size=(N, D)), torch.float32) for _ in range(2)) if s0 else (None, None))
        self.dones = torch.as_tensor((g.random((T, N)) < done_p).astype(np.uint8)) if done_p else None
        self.lengths = torch.as_tensor(g.integers(0, T + 1, N).astype(np.int32)) if ragged else None
        if ragged and N > 1:
            self.lengths[0], self.lengths[1] = T, 0

    def kw(self):
        n = lambda t: None if t is None else t.numpy()  # noqa: E731
        return dict(s0=f64(self.s0), dones=n(self.dones), lengths=n(self.lengths))

    def place(self, *xs):
        """Matrices on the GPU: side by side in one product's output, dense, sequences first, or one value further apart."""
        T, N, D = self.T, self.N, self.D
        if self.layout == "side":
            wide = torch.cat([x.cuda() for x in xs], 2)
            return [wide[..., i * D:(i + 1) * D] for i in range(len(xs))]
        if self.layout == "dense":
            return [x.cuda() for x in xs]
        if self.layout == "batch_first":
            return [x.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2) for x in xs]
        assert self.layout == "odd"
        out = []
        for x in xs:
            wide = torch.full((T, N, D + 1), float("nan"), dtype=x.dtype, device="cuda")
            wide[..., 1:] = x.cuda()
            out.append(wide[..., 1:])
        return out

    def empty(self, count):
        return self.place(*(torch.full((self.T, self.N, self.D), float("nan"), dtype=self.dtype) for _ in range(count)))

    def rec(self, rx):
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        return rx.GatedRec(self.dtype, self.T, self.N, self.D, dev(self.dones), dev(self.lengths))

    def state(self):
        return torch.full((self.N, self.D), float("nan"), device="cuda")

    def forward(self, rx):
        gr = self.rec(rx)
        x, g = self.place(self.x, self.g)
        (h,), s = self.empty(1), self.state()
        rx.rslx_gated_recurrence(gr, x, g, None if self.s0 is None else self.s0.cuda(), h, s, rx.workspace(rx.rslx_gated_recurrence_workspace_bytes(gr)))
        return h, s

    def backward(self, rx):
        gr = self.rec(rx)
        x, g, dh = self.place(self.x, self.g, self.dh)
        (dx, dg), ds0 = self.empty(2), self.state()
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        rx.rslx_gated_recurrence_backward(gr, x, g, dev(self.s0), dh, dev(self.ds_last), dx, dg, ds0,
                                          rx.workspace(rx.rslx_gated_recurrence_backward_workspace_bytes(gr)))
        return dx, dg, ds0

    def check_forward(self, h, s):
        x, g = f64(self.x), f64(self.g)
        ref, last, _ = ogr.forward(x, g, **self.kw())
        _, e, e_last = ogr.sizes(x, g, each=self.step, **self.kw())
        lost = self.T * 2.0 ** -126 * (1 + np.abs(x).max())
        check("h", h, ref, rounding(self.dtype, ref) + e + lost)
        check("s_last", s, last, e_last + lost)

    def check_backward(self, dx, dg, ds0):
        x, g, dh, kw = f64(self.x), f64(self.g), f64(self.dh), self.kw()
        f, rest = ogr.gates(g)
        ref = ogr.backward(x, g, dh, f64(self.ds_last), **kw)
        m, e, _ = ogr.sizes(x, g, each=self.step, **kw)
        entered = ogr.forward(np.abs(x), g, None if self.s0 is None else np.abs(f64(self.s0)), kw["dones"], kw["lengths"])[2]
        e_in = np.concatenate([np.zeros((1, self.N, self.D)), e[:-1]])
        # the walk from the end, over absolute values and over errors
        T = self.T
        md, ed = np.zeros_like(x), np.zeros_like(x)
        d = np.zeros((self.N, self.D)) if self.ds_last is None else np.abs(f64(self.ds_last))
        r = 0 * d
        for t in range(T - 1, -1, -1):
            here = ogr._there(t, kw["lengths"])
            keep = 1.0 if kw["dones"] is None else 1.0 - kw["dones"][t][:, None]
            md[t] = d * keep + np.abs(dh[t])
            ed[t] = r * keep + self.step * md[t]
            d, r = np.where(here, f[t] * md[t], d), np.where(here, f[t] * (ed[t] + self.step * md[t]), r)
        check("dx", dx, ref[0], rounding(self.dtype, ref[0]) + rest * (ed + self.step * md))
        diff = np.abs(ogr.forward(x, g, **kw)[2] - x)
        check("dg", dg, ref[1], rounding(self.dtype, ref[1]) + f * rest * (diff * (ed + 2 * self.step * md) + md * (e_in + 3 * U * (entered + np.abs(x)))))
        check("ds0", ds0, ref[2], r + self.step * d + 1e-37)


SIZES = [(1, 1, 1), (1, 5, 24), (2, 3, 64), (3, 2, 7), (24, 9, 256), (31, 3, 33), (32, 2, 128), (33, 2, 40), (64, 1, 65), (129, 2, 48), (255, 1, 20),
         (257, 3, 16), (513, 2, 72), (1025, 1, 8), (2100, 2, 64), (5000, 1, 12)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,N,D", SIZES)
def test_forward_and_backward(rx, T, N, D, dtype):
    c = Case(T * 7 + D, T, N, D, dtype, done_p=0.03, s0=True)
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [2, 3, 5, 6, 7, 66, 69, 129, 131])
def test_last_channels(rx, dtype, D):
    """Rows whose last piece is one, two or three values, with NaN on both sides of the row; episodes that end, sequences that are shorter."""
    for ragged in (False, True):
        c = Case(D, 75, 6, D, dtype, done_p=0.05, ragged=ragged, layout="odd")
        c.check_forward(*c.forward(rx))
        c.check_backward(*c.backward(rx))


@pytest.mark.parametrize("layout", ["side", "dense", "batch_first", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [6, 100, 700])
def test_ragged_and_layouts(rx, T, dtype, layout):
    c = Case(T, T, 6, 40, dtype, done_p=0.05, s0=T != 100, ragged=True, layout=layout)
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))


@pytest.mark.parametrize("T,N,D", [(24, 700, 256), (24, 1, 8192), (300, 300, 128), (3000, 3, 1024)])
def test_wide(rx, T, N, D):
    c = Case(T, T, N, D, "bf16", done_p=0.01, s0=False)
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))


@pytest.mark.parametrize("T", [0, 1, 3])
def test_no_steps_and_no_sequences(rx, T):
    c = Case(1, T, 4, 10, s0=True)
    c.lengths = torch.zeros(4, dtype=torch.int32)
    h, s = c.forward(rx)
    assert torch.equal(h, torch.zeros_like(h)) and torch.equal(s.cpu(), c.s0)
    dx, dg, ds0 = c.backward(rx)
    assert torch.equal(dx, torch.zeros_like(dx)) and torch.equal(dg, torch.zeros_like(dg)) and torch.equal(ds0.cpu(), c.ds_last)
    c.lengths = torch.tensor([-3, T + 5, 0, T], dtype=torch.int32)
    c.check_forward_lengths = None
    h2, s2 = c.forward(rx)
    c.lengths = torch.tensor([0, T, 0, T], dtype=torch.int32)
    h3, s3 = c.forward(rx)
    assert torch.equal(h2, h3) and torch.equal(s2, s3)
    e = Case(1, T, 0, 10, s0=False)
    h, s = e.forward(rx)
    assert h.numel() == 0 and s.numel() == 0


def test_states_may_be_left_out_or_shared(rx):
    c = Case(3, 70, 5, 36, done_p=0.05)
    gr, (x, g) = c.rec(rx), c.place(c.x, c.g)
    ws = rx.workspace(rx.rslx_gated_recurrence_workspace_bytes(gr))
    h, s = c.forward(rx)
    h2, s2 = c.empty(1)[0], c.s0.cuda()
    rx.rslx_gated_recurrence(gr, x, g, s2, h2, s2, ws)
    assert torch.equal(h, h2) and torch.equal(s, s2)
    rx.rslx_gated_recurrence(gr, x, g, c.s0.cuda(), h2, None, ws)
    assert torch.equal(h, h2)


def test_two_halves_are_the_whole(rx):
    c = Case(11, 300, 4, 24, done_p=0.02)
    h, s = c.forward(rx)
    a, b = Case(11, 300, 4, 24, done_p=0.02), Case(11, 300, 4, 24, done_p=0.02)
    for part, sl in ((a, slice(0, 133)), (b, slice(133, 300))):
        part.x, part.g, part.dones = c.x[sl], c.g[sl], c.dones[sl]
        part.T = part.x.shape[0]
    ha, sa = a.forward(rx)
    b.s0 = sa.cpu()
    hb, sb = b.forward(rx)
    e = ogr.sizes(f64(c.x), f64(c.g), each=2 * c.step, **c.kw())
    check("h", torch.cat([ha, hb]), f64(h), e[1])
    check("s", sb, f64(s), e[2] + 1e-37)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,D", [(1, 1), (64, 256), (300, 33), (4096, 24)])
def test_step(rx, N, D, dtype):
    c = Case(N, 1, N, D, dtype)
    gr, (x, g) = c.rec(rx), c.place(c.x, c.g)
    reset = torch.as_tensor((np.random.default_rng(1).random(N) < 0.3).astype(np.uint8))
    for flags in (None, reset):
        s0 = f64(c.s0) if flags is None else f64(c.s0) * (1 - flags.numpy()[:, None])
        ref, last, _ = ogr.forward(f64(c.x), f64(c.g), s0)
        m = ogr.sizes(f64(c.x), f64(c.g), s0)[0]
        h, s_in, s_out = c.empty(1)[0], c.s0.cuda(), c.state()
        rx.rslx_gated_recurrence_step(gr, x, g, None if flags is None else flags.cuda(), s_in, s_out, h)
        check("h", h, ref, rounding(c.dtype, ref) + c.step * m)
        check("s_out", s_out, last, c.step * m[0] + 1e-37)
        rx.rslx_gated_recurrence_step(gr, x, g, None if flags is None else flags.cuda(), s_in, s_in, x)       # both in place
        assert torch.equal(s_in, s_out) and torch.equal(x, h)
        x, g = c.place(c.x, c.g)
    ref = ogr.forward(f64(c.x), f64(c.g))[0]
    rx.rslx_gated_recurrence_step(gr, x, g, None, None, s_out, h)
    check("h", h, ref, rounding(c.dtype, ref) + c.step * np.abs(ref))


@pytest.mark.parametrize("T", [5, 200, 1500])
def test_what_is_not_finite_stays_in_its_episode(rx, T):
    """A step's values reach no earlier step and no other episode, channel or sequence; behind the length nothing is looked at."""
    c = Case(T, T, 4, 16, s0=True)
    cut, bad = T // 2, T // 2 - 1
    c.dones = torch.zeros(T, 4, dtype=torch.uint8)
    c.dones[cut - 1 if cut - 1 > bad else cut] = 1
    end = cut - 1 if cut - 1 > bad else cut
    c.lengths = torch.tensor([T, T, T - 1, T], dtype=torch.int32)
    clean = c.forward(rx), c.backward(rx)
    for value in (float("nan"), float("inf"), -float("inf")):
        d = Case(T, T, 4, 16, s0=True)
        d.dones, d.lengths = c.dones, c.lengths
        d.x[bad, 1, 3] = value
        d.x[T - 1, 2], d.g[T - 1, 2], d.dh[T - 1, 2] = value, float("nan"), value
        (h, s), (dx, dg, ds0) = d.forward(rx), d.backward(rx)
        touched = torch.zeros(T, 4, 16, dtype=torch.bool, device="cuda")
        touched[bad:end + 1, 1, 3] = True
        assert torch.equal(h[~touched], clean[0][0][~touched]) and torch.equal(s, clean[0][1])
        assert not torch.isfinite(h[touched]).any()
        assert torch.equal(dx, clean[1][0]) and torch.equal(ds0, clean[1][2])        # x has a part in dg alone
        assert torch.equal(dg[~touched], clean[1][1][~touched])
        e = Case(T, T, 4, 16, s0=True)
        e.dones, e.lengths = c.dones, c.lengths
        e.dh[bad, 1, 3] = value
        dx, dg, ds0 = e.backward(rx)
        touched = torch.zeros(T, 4, 16, dtype=torch.bool, device="cuda")
        touched[:bad + 1, 1, 3] = True
        assert torch.equal(dx[~touched], clean[1][0][~touched]) and torch.equal(dg[~touched], clean[1][1][~touched])
        assert not torch.isfinite(dx[touched]).any()


def test_gates_at_their_ends(rx):
    """g = inf holds the state, far below zero x comes in as it is; 1 - f keeps its digits next to one."""
    T, N, D = 40, 2, 8
    c = Case(5, T, N, D)
    c.g[:] = float("inf")
    h, s = c.forward(rx)
    assert torch.equal(h.cpu(), c.s0.expand(T, N, D)) and torch.equal(s.cpu(), c.s0)
    dx, dg, ds0 = c.backward(rx)
    assert not dx.any() and not dg.any()
    for value in (-float("inf"), -1000.0, -88.0):
        c.g[:] = value
        h, s = c.forward(rx)
        check("h", h, f64(c.x), 4 * U * np.abs(f64(c.x)) + 2.0 ** -125 * (1 + np.abs(f64(c.s0)).max()))
    c = Case(6, T, N, D, s0=False)
    c.g[:] = 30.0                                               # 1 - f = 1e-13
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))
    for value in (-90.0, 90.0, -104.0, 104.0):
        c.g[:] = value
        c.check_forward(*c.forward(rx))


def test_gradient_against_differences(rx):
    T, N, D = 9, 2, 3
    c = Case(8, T, N, D, done_p=0.2)
    dx, dg, ds0 = c.backward(rx)
    kw = c.kw()
    x, g, s0 = f64(c.x), f64(c.g), f64(c.s0)

    def loss(x, g, s0):
        h, last, _ = ogr.forward(x, g, s0, kw["dones"])
        return (h * f64(c.dh)).sum() + (last * f64(c.ds_last)).sum()
    for got, k in ((dx, 0), (dg, 1), (ds0, 2)):
        base = [x, g, s0]
        ref = np.zeros_like(base[k])
        for i in np.ndindex(ref.shape):
            up, down = [b.copy() for b in base], [b.copy() for b in base]
            up[k][i] += 1e-5
            down[k][i] -= 1e-5
            ref[i] = (loss(*up) - loss(*down)) / 2e-5
        # differences: the third derivative's part (1e-10) and rounding (1e-16 of a loss of about 50 over 2e-5)
        check("gradient", got, ref, 1e-9 + 200 * U * np.abs(ref) + 50 * U)


def test_graph_replays(rx):
    """Both directions in one captured graph, replayed between eager calls, with new inputs each time."""
    cases = [Case(s, 600, 3, 40, "bf16", done_p=0.02) for s in range(3)]
    c = cases[0]
    gr, (x, g, dh) = c.rec(rx), c.place(c.x, c.g, c.dh)
    s0, ds = c.s0.cuda(), c.ds_last.cuda()
    ws, wb = rx.workspace(rx.rslx_gated_recurrence_workspace_bytes(gr)), rx.workspace(rx.rslx_gated_recurrence_backward_workspace_bytes(gr))
    h, dx, dg = c.empty(3)
    s, ds0 = c.state(), c.state()

    def both():
        rx.rslx_gated_recurrence(gr, x, g, s0, h, s, ws)
        rx.rslx_gated_recurrence_backward(gr, x, g, s0, dh, ds, dx, dg, ds0, wb)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in (1, 2, 0, 1):
        for to, new in ((x, cases[k].x), (g, cases[k].g), (dh, cases[k].dh), (s0, cases[k].s0), (ds, cases[k].ds_last)):
            to.copy_(new.cuda())
        for t in (h, s, dx, dg, ds0):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h, s, dx, dg, ds0)]
        both()
        for a, b in zip(got, (h, s, dx, dg, ds0)):
            assert torch.equal(a, b)


def test_the_same_inputs_give_the_same_bits(rx):
    c = Case(2, 900, 3, 70, "fp16", done_p=0.01, ragged=True)
    for run in (c.forward, c.backward):
        first = run(rx)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, run(rx)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [7, 90, 300])
def test_rows_shared_by_sequences_or_steps(rx, T, dtype):
    """Inputs whose rows are the same memory for every sequence, or for every step: the gradients come for each."""
    c = Case(T, T, 5, 36, dtype, done_p=0.05)
    c.x, c.g, c.dh = c.x[:, :1].expand(T, 5, 36), c.g[:1].expand(T, 5, 36), c.dh[:1, :1].expand(T, 5, 36)

    def place(*xs):
        if all(0 in x.stride() for x in xs):
            return [x[tuple(slice(None) if s else slice(1) for s in x.stride())].contiguous().cuda().expand(x.shape) for x in xs]
        return [x.contiguous().cuda() for x in xs]
    c.place = place
    assert 0 in c.place(c.x)[0].stride()
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))


def test_two_streams_at_once(rx):
    """Calls on two streams, each with its own workspace and outputs, give what they give alone."""
    cases = [Case(20, 1500, 3, 64, "bf16", done_p=0.01), Case(21, 900, 5, 100, "fp32", done_p=0.01)]
    alone = [(c.forward(rx), c.backward(rx)) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append((c.forward(rx), c.backward(rx)))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            for x, y in zip(a, b):
                assert all(torch.equal(p, q) for p, q in zip(x, y))
