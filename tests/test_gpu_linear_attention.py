"""Linear attention with a decay for each head on the GPU against the step-by-step recurrence in fp64."""
import numpy as np
import pytest
import torch

from oracle import linear_attention as ola
from sequence_util import Attention, TYPES, U, check, f64, rounding, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


# T, N, H, Dk, Dv: single steps, whole and broken chunks, widths of one to all, both sides of every tile
SIZES = [(1, 1, 1, 1, 1), (2, 3, 2, 5, 7), (15, 2, 2, 16, 16), (16, 2, 1, 32, 32), (17, 3, 2, 33, 40), (24, 5, 4, 64, 64), (33, 2, 3, 64, 65),
         (48, 1, 2, 128, 128), (40, 2, 1, 100, 36), (31, 2, 2, 24, 20), (64, 1, 1, 8, 128), (20, 2, 2, 128, 3)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,N,H,Dk,Dv", SIZES)
def test_forward(rx, T, N, H, Dk, Dv, dtype):
    c = Attention(T * 131 + Dk, T, N, H, Dk, Dv, dtype, done_p=0.1, ragged=True)
    c.check_forward(*c.run_forward(rx))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,N,H,Dk,Dv", SIZES)
def test_backward(rx, T, N, H, Dk, Dv, dtype):
    c = Attention(T * 137 + Dv, T, N, H, Dk, Dv, dtype, done_p=0.1, ragged=True)
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("done_p", [0.0, 0.02, 1.0])
@pytest.mark.parametrize("s0,ragged", [(True, False), (False, False), (False, True)])
def test_episodes_lengths_and_start_states(rx, done_p, s0, ragged):
    c = Attention(11, 50, 6, 2, 20, 12, "fp32", done_p=done_p, s0=s0, ragged=ragged)
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("layout", ["batch_first", "head_first", "odd", "shared_key"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_layouts(rx, layout, dtype):
    c = Attention(12, 37, 3, 4, 32, 48, dtype, done_p=0.05, ragged=True, layout=layout)
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


# few heads: the sequences are walked in pieces
@pytest.mark.parametrize("T,N,H,Dk,Dv,dtype", [(128, 1, 1, 16, 16, "fp32"), (200, 2, 1, 33, 64, "fp16"), (1000, 1, 2, 64, 32, "fp32"),
                                               (777, 3, 2, 40, 72, "bf16"), (2500, 2, 1, 128, 64, "bf16")])
@pytest.mark.parametrize("ragged", [False, True])
def test_pieces(rx, T, N, H, Dk, Dv, dtype, ragged):
    c = Attention(T, T, N, H, Dk, Dv, dtype, done_p=0.005, ragged=ragged)
    c.on_gpu(rx)
    assert rx.rslx_linear_attention_workspace_bytes(c.la) > 256
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


def test_long_memory_keeps_its_digits(rx):
    """20 000 steps of a memory that hardly forgets: rounding must not add up over the chunks."""
    c = Attention(13, 20000, 1, 2, 8, 8, "fp32", s0=True, decays=[-1e-5, -3e-4])
    o, s = c.run_forward(rx)
    ro, rs = ola.forward(*c.args(), **c.kw())
    for got, ref in ((o, ro), (s, rs)):
        got = f64(got)
        # a random walk of the roundings instead of their sum: sqrt(2 T) u of the terms' root sum of squares, which is the result's size
        assert np.linalg.norm(got - ref) <= np.sqrt(2 * 20000 + 64) * U * np.linalg.norm(ref)


@pytest.mark.parametrize("log_decay", [0.0, -1e-7, -3.0, -200.0, -1e30, float("-inf")])
def test_decays_from_everything_to_nothing(rx, log_decay):
    c = Attention(14, 40, 2, 1, 12, 20, "fp32", done_p=0.05, decays=[log_decay])
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("T", [0, 1])
def test_no_step_and_one_step(rx, T):
    c = Attention(15, T, 3, 2, 8, 16, "fp32")
    o, s = c.run_forward(rx)
    c.check_forward(o, s)
    c.check_backward(*c.run_backward(rx))
    if T == 0:
        assert torch.equal(s.cpu(), c.s0)


def test_rows_behind_a_sequence_are_not_looked_at(rx):
    c = Attention(16, 45, 4, 2, 16, 24, "bf16", done_p=0.05, ragged=True)
    clean = [x.clone() for x in (*c.run_forward(rx), *c.run_backward(rx))]
    for n in range(c.N):
        for x in (c.q, c.k, c.v, c.do):
            x[int(c.lengths[n]):, n] = float("nan")
    for a, b in zip(clean, (*c.run_forward(rx), *c.run_backward(rx))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("T", [40, 200])
def test_what_is_not_finite_stays_where_it_belongs(rx, name, value, T):
    c = Attention(17, T, 3, 2, 8, 12, "fp32", done_p=0.05)
    for t, n, h in ((3, 0, 0), (T // 2, 1, 1), (T - 1, 2, 0)):
        getattr(c, name)[t, n, h, 2] = value
    c.dones[:, 2] = 0
    c.dones[T // 2 + 5, 1] = 1
    c.dones[9, 0] = 1
    more = dict(do=f64(c.do), ds_last=f64(c.ds_last))
    ref = ola.forward(*c.args(), **c.kw()) + ola.backward(*c.args(), **c.kw(), **more)
    got = c.run_forward(rx) + c.run_backward(rx)
    for what, r, x in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), ref, got):
        x = f64(x)
        fine = np.isfinite(r)
        assert np.array_equal(np.isfinite(x), fine), (what, int((np.isfinite(x) != fine).sum()))
        # sizes of sums of finite terms: within a few hundred roundings of the largest
        assert np.abs(x[fine] - r[fine]).max(initial=0) <= c.roundings * U * 40 * max(1.0, np.abs(r[fine]).max(initial=0)), what


# 16 bits: a wavefront per tile of columns, with the rows of wide keys shared by a workgroup, or by itself
@pytest.mark.parametrize("T,N,H,Dk,Dv,dtype", [(700, 2, 2, 128, 128, "bf16"), (333, 3, 1, 100, 97, "fp16"), (130, 2, 1, 72, 128, "bf16")])
def test_wide_heads_in_pieces(rx, T, N, H, Dk, Dv, dtype):
    c = Attention(T + 1, T, N, H, Dk, Dv, dtype, done_p=0.01, ragged=True)
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Dk,Dv", [(40, 128, 100), (200, 128, 128), (70, 40, 64)])
def test_what_is_not_finite_in_16_bits(rx, name, dtype, T, Dk, Dv):
    c = Attention(T + 2, T, 3, 2, Dk, Dv, dtype, done_p=0.05)
    for t, n, h, value in ((3, 0, 0, float("inf")), (T // 2, 1, 1, float("nan")), (T - 1, 2, 0, float("-inf"))):
        getattr(c, name)[t, n, h, 2] = value
    c.dones[:, 2] = 0
    c.dones[T // 2 + 5, 1] = 1
    c.dones[9, 0] = 1
    more = dict(do=f64(c.do), ds_last=f64(c.ds_last))
    ref = ola.forward(*c.args(), **c.kw()) + ola.backward(*c.args(), **c.kw(), **more)
    got = c.run_forward(rx) + c.run_backward(rx)
    for what, r, x in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), ref, got):
        x = f64(x)
        fine = np.isfinite(r)
        assert np.array_equal(np.isfinite(x), fine), (what, int((np.isfinite(x) != fine).sum()))
        # the output's own rounding, and the products' (2^-17 of a term at most, and terms of 40 times the largest result in all)
        size = max(1.0, np.abs(r[fine]).max(initial=0))
        assert np.abs(x[fine] - r[fine]).max(initial=0) <= (torch.finfo(c.dtype).eps / 2 + 40 * 2.0 ** -17 + c.roundings * U * 40) * size, what


def test_two_calls_are_one(rx):
    c = Attention(18, 60, 4, 2, 24, 40, "fp32", done_p=0.05)
    g, la = c.on_gpu(rx)
    state, parts = g["s0"].clone(), []
    for a, b in ((0, 23), (23, 24), (24, 60)):
        part = rx.LinearAttn(c.dtype, b - a, c.N, c.H, c.Dk, c.Dv, la.log_decay, c.scale, la.dones[a:b].contiguous())
        o = torch.empty(b - a, c.N, c.H, c.Dv, device="cuda")
        rx.rslx_linear_attention(part, g["q"][a:b], g["k"][a:b], g["v"][a:b], state, o, state, None)       # in place
        parts.append(o)
    c.check_forward(torch.cat(parts), state)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,H,Dk,Dv", [(1, 1, 1, 1), (3, 2, 5, 7), (64, 4, 32, 32), (33, 3, 64, 64), (5, 2, 128, 128), (7, 1, 100, 36), (4, 5, 17, 128),
                                       (2, 2, 128, 65), (130, 1, 20, 2)])
def test_step(rx, N, H, Dk, Dv, dtype):
    for reset_p, has_state, layout in ((0.3, True, "dense"), (0.0, True, "odd"), (0.5, False, "dense")):
        c = Attention(N * 7 + Dk, 1, N, H, Dk, Dv, dtype, done_p=reset_p, layout=layout)
        reset, c.dones = c.dones, None
        g, la = c.on_gpu(rx)
        o, s = c.empty(Dv), c.state()
        s_in = g["s0"] if has_state else None
        rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], None if reset is None else reset.cuda(), s_in, s, o)
        args = (f64(c.q)[0], f64(c.k)[0], f64(c.v)[0], f64(c.log_decay), c.scale)
        kw = dict(s_in=f64(c.s0) if has_state else None, reset=None if reset is None else reset[0].numpy())
        ro, rs = ola.step(*args, **kw)
        mo, ms = ola.step(*(np.abs(x) if isinstance(x, np.ndarray) and x.ndim == 3 else x for x in args),
                          **dict(kw, s_in=None if not has_state else np.abs(kw["s_in"])))
        # a product and two roundings per element of the state, then a sum of Dk products
        check("o", o[0], ro, rounding(c.dtype, ro) + (Dk + 12) * U * mo)
        check("s_out", s, rs, 6 * U * ms)
        if has_state:                                          # in place, the same bits
            s2 = g["s0"].clone()
            rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], None if reset is None else reset.cuda(), s2, s2, o)
            assert torch.equal(s, s2)


def test_steps_are_the_sequence(rx):
    c = Attention(19, 20, 5, 3, 16, 32, "fp32", done_p=0.1)
    g, la = c.on_gpu(rx)
    one = rx.LinearAttn(c.dtype, 1, c.N, c.H, c.Dk, c.Dv, la.log_decay, c.scale)
    state, o = g["s0"].clone(), torch.empty(c.T, c.N, c.H, c.Dv, device="cuda")
    for t in range(c.T):
        reset = None if t == 0 else la.dones[t - 1]
        rx.rslx_linear_attention_step(one, g["q"][t:t + 1], g["k"][t:t + 1], g["v"][t:t + 1], reset, state, state, o[t:t + 1])
    state[la.dones[-1].bool()] = 0
    c.check_forward(o, state)


def test_a_poisoned_state_ends_with_its_episode(rx):
    c = Attention(20, 1, 4, 2, 8, 8, "fp32")
    g, la = c.on_gpu(rx)
    s = g["s0"].clone()
    s[1] = float("nan")
    o = c.empty(8)
    rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda"), s, s, o)
    assert torch.isfinite(o).all() and torch.isfinite(s).all()


def test_same_inputs_same_bits(rx):
    c = Attention(21, 500, 2, 2, 64, 64, "bf16", done_p=0.01)
    first = [x.clone() for x in (*c.run_forward(rx), *c.run_backward(rx))]
    for a, b in zip(first, (*c.run_forward(rx), *c.run_backward(rx))):
        assert torch.equal(a, b)


def test_rows_further_apart_than_32_bits_reach(rx):
    T, N, H, D = 3, 1, 2, 16
    far = (1 << 31) + 48                                       # elements from step to step; two bytes each
    big = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    c = Attention(22, T, N, H, D, D, "bf16")
    at = lambda offset: torch.as_strided(big, (T, N, H, D), (far, H * D, D, 1), offset)  # noqa: E731
    views = [at(64 * i) for i in range(4)]
    for x, y in zip(views, (c.q, c.k, c.v, c.do)):
        x.copy_(y)
    g, la = c.on_gpu(rx)
    o, s = at(64 * 4), c.state()
    rx.rslx_linear_attention(la, *views[:3], g["s0"], o, s, None)
    c.check_forward(o, s)
    dq, dk, dv, ds0 = at(64 * 5), at(64 * 6), at(64 * 7), c.state()
    rx.rslx_linear_attention_backward(la, *views[:3], g["s0"], views[3], g["ds_last"], dq, dk, dv, ds0, None)
    c.check_backward(dq, dk, dv, ds0)


def test_another_stream_and_a_graph(rx):
    c = Attention(23, 300, 2, 2, 32, 64, "fp32", done_p=0.01)
    g, la = c.on_gpu(rx)
    want = [x.clone() for x in (*c.run_forward(rx), *c.run_backward(rx))]
    o, s, dq, dk, dv, ds0 = c.empty(c.Dv), c.state(), c.empty(c.Dk), c.empty(c.Dk), c.empty(c.Dv), c.state()
    wf = rx.workspace(rx.rslx_linear_attention_workspace_bytes(la))
    wb = rx.workspace(rx.rslx_linear_attention_backward_workspace_bytes(la))

    def both():
        rx.rslx_linear_attention(la, g["q"], g["k"], g["v"], g["s0"], o, s, wf)
        rx.rslx_linear_attention_backward(la, g["q"], g["k"], g["v"], g["s0"], g["do"], g["ds_last"], dq, dk, dv, ds0, wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    outs = (o, s, dq, dk, dv, ds0)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):                                         # every replay against the eager results
        for x in outs:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        both()
        torch.cuda.synchronize()


def test_gradients_are_differences_of_the_forward_call(rx):
    c = Attention(24, 40, 2, 2, 16, 16, "fp32", done_p=0.1)
    dq, dk, dv, ds0 = c.run_backward(rx)
    g, la = c.g, c.la

    def loss(**kw):
        a = dict(g, **kw)
        o, s = c.empty(c.Dv), c.state()
        rx.rslx_linear_attention(la, a["q"], a["k"], a["v"], a["s0"], o, s, None)
        return float((o.double() * g["do"].double()).sum() + (s.double() * g["ds_last"].double()).sum())

    r = np.random.default_rng(5)
    for name, grad in (("q", dq), ("k", dk), ("v", dv), ("s0", ds0)):
        # the loss is linear in each of q, k, v, s0: one long step is exact but for rounding (the loss is a sum of about 4000 outputs
        # of size 10, each 1e-6 of its size off, over a step of 1)
        d = torch.as_tensor(r.normal(size=g[name].shape), dtype=torch.float32, device="cuda")
        got = float((grad.double() * d.double()).sum())
        want = (loss(**{name: g[name] + d}) - loss(**{name: g[name] - d})) / 2
        assert abs(got - want) <= 1e-2 + 1e-5 * abs(want), (name, got, want)


def test_trace_names_the_launches(rx):
    c = Attention(25, 256, 1, 2, 16, 16, "fp32")
    c.run_forward(rx)
    rx.rslx_trace_begin(64)
    c.run_forward(rx)
    c.run_backward(rx)
    torch.cuda.synchronize()
    names = [r[0] for r in rx.rslx_trace_end()]
    assert names == ["linear_attention_states", "linear_attention_join", "linear_attention_walk"] * 2
