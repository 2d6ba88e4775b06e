"""Muon step on the GPU against fp64.

Bounds, in the Frobenius norm.  A product of held operands loses e = 16 u of the norms of its factors (u = 2^-24: three times 2^-22 = 12 u for what pairs of fp16
leave out, the sum's roundings of either sign another 4), |X Y| <= |X|_F |Y|_2.  With |X|_2 <= 1.21, A = X X^T <= 1.47 and B <= 3.45, one step adds
(4.775 + 2 * 2.0315 * 1.47) * 1.21^2 e (through A), 2.0315 * 1.47 * 1.21^2 e (A^2) and 3.45 * 1.21 e (B X) of |X|_F, 25 e together, and each later
step enlarges it by at most oracle.muon.steepest.
"""
import numpy as np
import pytest
import torch

from oracle import muon as om
from sequence_util import U, check, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


def _bound(u, steps):
    trace = []
    om.orthogonalize(u, steps, trace)
    e = 0.0
    for x in trace:
        s = np.linalg.svd(x, compute_uv=False)
        e = e * om.steepest(s) + 25 * 16 * U * np.linalg.norm(x)
    return e


def _matrices(seed, shapes, spread=True):
    g = np.random.default_rng(seed)
    f = lambda x: torch.as_tensor(x).float().cuda()  # noqa: E731
    out = []
    for a, b in shapes:
        grad = g.normal(size=(a, b)) * 1e-3
        out.append((f(g.normal(size=(a, b)) * 0.1), f(grad), f(g.normal(size=(a, b)) * 5e-3), float(np.float32(np.sqrt(max(1, b / a))))))
    return out


def _check(name, w, grad, m, scale, w_out, m_out, cfg):
    lr, beta, nesterov, decay, steps = cfg
    w, grad, m = (None if t is None else f64(t) for t in (w, grad, m))
    ref_w, ref_m, x, u = om.step(0 if w is None else w, grad, 0 if m is None else m, lr, beta, nesterov, decay, steps, scale)
    if m_out is not None:
        check(name + " m", m_out, ref_m, 2 * U * (np.abs(grad) + (0 if m is None else beta * np.abs(m))))
    bound = abs(lr) * scale * (_bound(u, steps) + 4 * U * np.linalg.norm(x)) + (0 if w is None else 4 * U * np.linalg.norm(w))
    off = np.linalg.norm(f64(w_out) - ref_w)
    assert off <= bound, (name, off, bound)
    return off / bound


SHAPES = [(1, 1), (1, 7), (9, 1), (12, 128), (128, 12), (32, 32), (33, 31), (48, 512), (64, 64), (65, 130), (100, 30), (128, 128), (129, 127), (235, 512),
          (256, 512), (512, 256), (320, 777), (777, 333), (600, 600)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_one_matrix(rx, rows, cols):
    cfg = (0.02, 0.95, True, 0.01, 5)
    f32 = [float(np.float32(c)) for c in (0.02, 0.95)] + [True, float(np.float32(0.01)), 5]
    (w, grad, m, scale), = _matrices(rows * 1000 + cols, [(rows, cols)])
    w_out, m_out = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    mu = rx.Muon([(w, w_out, grad, m, m_out, scale)], *cfg[:1], momentum=cfg[1], nesterov=cfg[2], weight_decay=cfg[3], steps=cfg[4])
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    _check("step", w, grad, m, scale, w_out, m_out, f32)
    # the update alone: nothing kept, nothing decayed
    x = torch.full_like(w, float("nan"))
    mu = rx.Muon([(None, x, grad, None, None, 1.0)], -1.0, nesterov=False, steps=5)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    _check("update", None, grad, None, 1.0, x, None, (-1.0, f32[1], False, 0.0, 5))


@pytest.mark.parametrize("steps", [1, 2, 3, 6])
@pytest.mark.parametrize("nesterov", [False, True])
def test_steps_of_many_matrices_in_flat_buffers(rx, steps, nesterov):
    """Weights of two networks inside flat parameter buffers, in place; what lies between them stays."""
    shapes = [(48, 512), (512, 256), (256, 128), (128, 12), (235, 512), (512, 256), (256, 128), (128, 1)]
    n = sum(a * b + b for a, b in shapes)
    gen = torch.Generator("cuda").manual_seed(5)
    w, grad, m = (torch.randn(n, generator=gen, device="cuda") * k for k in (0.1, 1e-3, 5e-3))
    before = [t.clone() for t in (w, grad, m)]
    at, mats, views = 0, [], []
    for a, b in shapes:
        v = [t[at:at + a * b].view(a, b) for t in (w, grad, m)]
        views.append((at, a, b))
        mats.append((v[0], v[0], v[1], v[2], v[2], 1.5))
        at += a * b + b
    mu = rx.Muon(mats, 0.05, momentum=0.9, nesterov=nesterov, steps=steps)
    ws = rx.workspace(rx.rslx_muon_step_workspace_bytes(mu))
    rx.rslx_muon_step(mu, ws)
    cfg = (float(np.float32(0.05)), float(np.float32(0.9)), nesterov, 0.0, steps)
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    for at, a, b in views:
        part = [t[at:at + a * b].view(a, b) for t in before]
        _check("%dx%d" % (a, b), *part, 1.5, w[at:at + a * b].view(a, b), m[at:at + a * b].view(a, b), cfg)
        inside[at:at + a * b] = True
    assert torch.equal(w[~inside], before[0][~inside]) and torch.equal(m[~inside], before[2][~inside]) and torch.equal(grad, before[1])


def test_a_matrix_does_not_depend_on_its_company(rx):
    shapes = [(40, 70), (300, 200), (64, 64), (5, 300)]
    mats = _matrices(3, shapes)
    outs = [torch.empty_like(w) for w, *_ in mats]
    mu = rx.Muon([(w, o, g, m, None, s) for (w, g, m, s), o in zip(mats, outs)], 0.1)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    for (w, g, m, s), o in zip(mats, outs):
        alone = torch.empty_like(w)
        mu = rx.Muon([(w, alone, g, m, None, s)], 0.1)
        rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
        assert torch.equal(alone, o)


def test_equal_singular_values_keep_fp32s_digits(rx):
    """A rotation's singular values are equal: nothing is enlarged more than the result itself, and the bound is tight (about 1e-4; fp16 alone would be off by 1e-3)."""
    q = np.linalg.qr(np.random.default_rng(1).normal(size=(96, 96)))[0]
    u = torch.as_tensor(3e-4 * q).float().cuda()
    x = torch.empty_like(u)
    mu = rx.Muon([(None, x, u, None, None, 1.0)], -1.0, nesterov=False, steps=5)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    ref = om.orthogonalize(f64(u), 5)
    assert np.linalg.norm(f64(x) - ref) <= min(_bound(f64(u), 5), 3e-4 * np.linalg.norm(ref))


@pytest.mark.parametrize("size", [1e-30, 1e-3, 1.0, 1e18, 3e37])
def test_sizes_of_the_update(rx, size):
    """The update's size has no part in the result, from where squares vanish in fp32 to where they overflow."""
    g = torch.Generator("cuda").manual_seed(2)
    u = torch.randn(40, 90, generator=g, device="cuda")
    x = torch.empty_like(u)
    mu = rx.Muon([(None, x, u * size, None, None, 1.0)], -1.0, nesterov=False, steps=5)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    _check("size", None, u * size, None, 1.0, x, None, (-1.0, 0.0, False, 0.0, 5))


def test_zeros_and_what_is_not_finite(rx):
    mats = _matrices(7, [(30, 50), (30, 50), (64, 40), (20, 200)])
    zero, nan, inf = mats[0], mats[1], mats[2]
    zero[1].zero_(), zero[2].zero_()
    nan[1][3, 4] = float("nan")
    inf[1][5, 6] = float("inf")
    outs = [torch.empty_like(w) for w, *_ in mats]
    mu = rx.Muon([(w, o, g, m, None, s) for (w, g, m, s), o in zip(mats, outs)], 0.1)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    assert torch.equal(outs[0], mats[0][0])
    assert torch.isnan(outs[1]).all() and torch.isnan(outs[2]).all()
    _check("beside", *mats[3], outs[3], None, (float(np.float32(0.1)), float(np.float32(0.95)), True, 0.0, 5))


def test_low_rank(rx):
    """A gradient of rank 3: the other singular values are rounding's, and enlarged with it."""
    g = np.random.default_rng(4)
    u = torch.as_tensor(g.normal(size=(120, 3)) @ g.normal(size=(3, 80))).float().cuda()
    x = torch.empty_like(u)
    mu = rx.Muon([(None, x, u, None, None, 1.0)], -1.0, nesterov=False, steps=5)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    _check("low rank", None, u, None, 1.0, x, None, (-1.0, 0.0, False, 0.0, 5))


def test_no_matrices_and_graph_replays(rx):
    mu = rx.Muon([], 0.1)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    mats = _matrices(3, [(40, 70), (200, 100)])
    outs = [(torch.empty_like(w), torch.empty_like(w)) for w, *_ in mats]
    mu = rx.Muon([(w, o, g, m, mo, s) for (w, g, m, s), (o, mo) in zip(mats, outs)], 0.1)
    ws = rx.workspace(rx.rslx_muon_step_workspace_bytes(mu))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        rx.rslx_muon_step(mu, ws)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rx.rslx_muon_step(mu, ws)
    for k in range(3):
        for _, g, m, _ in mats:
            g.copy_(g.flip(0) * 1.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for o in outs for t in o]
        rx.rslx_muon_step(mu, ws)
        assert all(torch.equal(a, b) for a, b in zip(got, [t for o in outs for t in o]))
