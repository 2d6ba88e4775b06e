"""Arguments that the operators around a gated memory refuse, on the host, before anything is launched."""
import pytest
import torch

import paper_2509_10771_amd as rx
from paper_2509_10771_amd import binding as B

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors here are on the CPU; calls that are taken end at the launch only without a GPU")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
Z = torch.zeros


# ---- gated linear recurrence ------------------------------------------------------------------------------------------
def _rec(T=3, N=2, D=8, dtype=F32, **kw):
    return rx.GatedRec(dtype, T, N, D, **kw)


def _forward(gr, **kw):
    z = lambda: Z(gr.T, gr.N, gr.D, dtype=gr.dtype)  # noqa: E731
    a = dict(x=z(), g=z(), s0=None, h=z(), s_last=None, ws=None)
    a.update(kw)
    rx.rslx_gated_recurrence(gr, *(a[n] for n in ("x", "g", "s0", "h", "s_last", "ws")))


def _backward(gr, **kw):
    z = lambda: Z(gr.T, gr.N, gr.D, dtype=gr.dtype)  # noqa: E731
    a = dict(x=z(), g=z(), s0=None, dh=z(), ds_last=None, dx=z(), dg=z(), ds0=None, ws=None)
    a.update(kw)
    rx.rslx_gated_recurrence_backward(gr, *(a[n] for n in ("x", "g", "s0", "dh", "ds_last", "dx", "dg", "ds0", "ws")))


def test_recurrence_shapes_and_types():
    with pytest.raises(rx.RslxError, match="not one of"):
        _rec(dtype=torch.float64)
    with pytest.raises(rx.RslxError, match="D = 0"):
        rx.rslx_gated_recurrence_workspace_bytes(_rec(D=0))
    with pytest.raises(rx.RslxError, match="exceeds"):
        rx.rslx_gated_recurrence_workspace_bytes(_rec(N=1 << 16, D=1 << 15))
    with pytest.raises(rx.RslxError, match="too many"):
        rx.rslx_gated_recurrence_backward_workspace_bytes(_rec(T=1 << 20, N=1 << 16, D=1))
    with pytest.raises(rx.RslxError, match="too many"):
        rx.rslx_gated_recurrence_backward_workspace_bytes(_rec(T=129, N=1 << 16, D=1 << 12))
    with pytest.raises(rx.RslxError, match="more than 32 bits"):
        _rec(T=1 << 32)
    with pytest.raises(rx.RslxError, match="x is"):
        _forward(_rec(), x=Z(3, 2, 7))
    with pytest.raises(rx.RslxError, match="g is"):
        _forward(_rec(), g=Z(3, 2, 8, dtype=BF16))
    with pytest.raises(rx.RslxError, match="side by side"):
        _forward(_rec(), h=Z(3, 8, 2).transpose(1, 2))
    with pytest.raises(rx.RslxError, match="dones"):
        _rec(dones=Z(3, 2))
    with pytest.raises(rx.RslxError, match="lengths"):
        _rec(lengths=Z(3, dtype=torch.int32))
    with pytest.raises(rx.RslxError, match="s0 has"):
        _forward(_rec(), s0=Z(2, 7))
    with pytest.raises(rx.RslxError, match="s_last has"):
        _forward(_rec(), s_last=Z(2, 8, dtype=BF16))
    gr = _rec()
    gr.c.T = -1
    assert rx.lib.rslx_gated_recurrence_workspace_bytes(gr.c) == 0 and b"T = -1" in rx.lib.rslx_last_error()
    gr = _rec()
    gr.c.T = 2 ** 31 - 64
    assert rx.lib.rslx_gated_recurrence_workspace_bytes(gr.c) == 0
    gr = _rec()
    gr.c.dtype = 9
    with pytest.raises(rx.RslxError, match="unknown dtype"):
        _forward(gr)
    assert rx.lib.rslx_gated_recurrence_workspace_bytes(None) == 0
    assert rx.lib.rslx_gated_recurrence(None, None, None, None, None, None, None, 0, None) == 1


def test_recurrence_pointers():
    gr = _rec()
    v = gr.view("v", Z(3, 2, 8))
    assert rx.lib.rslx_gated_recurrence(gr.c, None, v, None, v, None, None, 0, None) == 1 and b"null x" in rx.lib.rslx_last_error()
    assert rx.lib.rslx_gated_recurrence(gr.c, v, v, None, None, None, None, 0, None) == 1 and b"null h" in rx.lib.rslx_last_error()
    half = B._CSeqView(v.data + 2, v.step, v.seq, 0)
    assert rx.lib.rslx_gated_recurrence(gr.c, half, v, None, v, None, None, 0, None) == 1 and b"not aligned to its type" in rx.lib.rslx_last_error()
    with pytest.raises(rx.RslxError, match="16-byte"):
        _forward(gr, s0=Z(17)[1:].view(2, 8))
    with pytest.raises(rx.RslxError, match="null s_out"):
        rx.rslx_gated_recurrence_step(_rec(T=1), Z(1, 2, 8), Z(1, 2, 8), None, None, None, Z(1, 2, 8))
    with pytest.raises(rx.RslxError, match="T = 1"):
        rx.rslx_gated_recurrence_step(_rec(T=2), Z(2, 2, 8), Z(2, 2, 8), None, None, Z(2, 8), Z(2, 2, 8))
    with pytest.raises(rx.RslxError, match="T = 1"):
        rx.rslx_gated_recurrence_step(_rec(T=1, dones=Z(1, 2, dtype=torch.uint8)), Z(1, 2, 8), Z(1, 2, 8), None, None, Z(2, 8), Z(1, 2, 8))
    with pytest.raises(rx.RslxError, match="reset"):
        rx.rslx_gated_recurrence_step(_rec(T=1), Z(1, 2, 8), Z(1, 2, 8), Z(2), None, Z(2, 8), Z(1, 2, 8))
    wrong = ((Z(2, 8), "needed"), (Z(1, 2, 4), "needed"), (Z(1, 2, 8, dtype=torch.float16), "needed"), (Z(1, 2, 16)[..., ::2], "side by side"))
    for name in ("x", "g", "h"):                              # the views of a step, each wrong in turn
        for t, word in wrong:
            rows = dict({n: Z(1, 2, 8) for n in ("x", "g", "h")}, **{name: t})
            with pytest.raises(rx.RslxError, match="^%s.* %s" % (name, word)):
                rx.rslx_gated_recurrence_step(_rec(T=1), rows["x"], rows["g"], None, None, Z(2, 8), rows["h"])
    for n, s in ((17, Z(17)), (16, Z(16, dtype=torch.float16))):
        for states in ((s, Z(2, 8)), (None, s)):
            with pytest.raises(rx.RslxError, match="s_(in|out) has %d values" % n):
                rx.rslx_gated_recurrence_step(_rec(T=1), Z(1, 2, 8), Z(1, 2, 8), None, *states, Z(1, 2, 8))


def test_recurrence_outputs_that_overlap():
    with pytest.raises(rx.RslxError, match="rows of h overlap"):
        _forward(_rec(), h=Z(3, 1, 8).expand(3, 2, 8))
    m = Z(3, 2, 8)
    with pytest.raises(rx.RslxError, match="h overlaps x"):
        _forward(_rec(), x=m, h=m)
    s = Z(40)
    with pytest.raises(rx.RslxError, match="s_last overlaps s0"):
        _forward(_rec(), s0=s[:16].view(2, 8), s_last=s[4:20].view(2, 8))
    with pytest.raises(rx.RslxError, match="s_last overlaps x"):
        _forward(_rec(), x=m, s_last=m.view(-1)[:16].view(2, 8))
    with pytest.raises(rx.RslxError, match="h overlaps s0"):
        _forward(_rec(), h=m, s0=m.view(-1)[16:32].view(2, 8))
    for a, b in (("dx", "x"), ("dg", "dh"), ("dx", "dg"), ("dg", "g")):
        with pytest.raises(rx.RslxError, match="%s overlaps %s" % (a, b)):
            _backward(_rec(), **{a: m, b: m})
    with pytest.raises(rx.RslxError, match="ds0 overlaps ds_last"):
        _backward(_rec(), ds0=s[:16].view(2, 8), ds_last=s[:16].view(2, 8))
    with pytest.raises(rx.RslxError, match="ds0 overlaps s0"):
        _backward(_rec(), ds0=s[:16].view(2, 8), s0=s[8:24].view(2, 8))
    dones = m.view(-1).view(torch.uint8)[:6].view(3, 2)
    with pytest.raises(rx.RslxError, match="h overlaps dones"):
        _forward(_rec(dones=dones), h=m)
    with pytest.raises(rx.RslxError, match="dx overlaps lengths"):
        _backward(_rec(lengths=m.view(-1).view(torch.int32)[2:4]), dx=m)
    step = lambda **kw: rx.rslx_gated_recurrence_step(_rec(T=1), *(  # noqa: E731
        dict(dict(x=Z(1, 2, 8), g=Z(1, 2, 8), reset=None, s_in=None, s_out=Z(2, 8), h=Z(1, 2, 8)), **kw)[n] for n in ("x", "g", "reset", "s_in", "s_out", "h")))
    one = Z(60)
    with pytest.raises(rx.RslxError, match="h overlaps x, and not row by row"):
        step(x=one[:16].view(1, 2, 8), h=one[4:20].view(1, 2, 8))
    with pytest.raises(rx.RslxError, match="s_out overlaps s_in"):
        step(s_in=one[:16].view(2, 8), s_out=one[4:20].view(2, 8))
    with pytest.raises(rx.RslxError, match="s_out overlaps g"):
        step(g=one[:16].view(1, 2, 8), s_out=one[:16].view(2, 8))
    with pytest.raises(rx.RslxError, match="h overlaps s_in"):
        step(s_in=one[:16].view(2, 8), h=one[:16].view(1, 2, 8))


def test_recurrence_workspace():
    for T in (1, 4096):
        gr = _rec(T=T)
        assert rx.rslx_gated_recurrence_workspace_bytes(gr) >= 256 and rx.rslx_gated_recurrence_backward_workspace_bytes(gr) >= 256
    with pytest.raises(rx.RslxError, match="workspace"):
        _backward(_rec(T=8192, N=4, D=1024, dtype=BF16))
    n = rx.rslx_gated_recurrence_backward_workspace_bytes(_rec(T=8192, N=1, D=8))
    with pytest.raises(rx.RslxError, match="workspace"):
        _backward(_rec(T=8192, N=1, D=8), ws=Z(n // 4, dtype=torch.uint8))       # (aligned rows are cut into half as many pieces as the query has to expect)
    with pytest.raises(rx.RslxError, match="workspace not 16-byte"):
        _backward(_rec(T=8192, N=1, D=8), ws=Z(n + 8, dtype=torch.uint8)[8:])


# ---- root-mean-square norm ----------------------------------------------------------------------------------------------
def test_norm_refusals():
    x, w = Z(4, 8), Z(8)
    with pytest.raises(rx.RslxError, match="residual is"):
        rx.rslx_rms_norm(x, Z(4, 7), w, 1e-5, None, Z(4, 8), None)
    with pytest.raises(rx.RslxError, match="total is"):
        rx.rslx_rms_norm(x, None, w, 1e-5, Z(4, 8, dtype=BF16), Z(4, 8), None)
    with pytest.raises(rx.RslxError, match="a matrix of float32"):
        rx.rslx_rms_norm(x.double(), None, w, 1e-5, None, Z(4, 8), None)
    with pytest.raises(rx.RslxError, match="columns"):
        rx.rslx_rms_norm(Z(1, 16385), None, None, 1e-5, None, Z(1, 16385), None)
    with pytest.raises(rx.RslxError, match="weight has"):
        rx.rslx_rms_norm(x, None, Z(7), 1e-5, None, Z(4, 8), None)
    with pytest.raises(rx.RslxError, match="null x, y or scales"):
        rx.rslx_rms_norm(x, None, w, 1e-5, None, None, None)
    with pytest.raises(rx.RslxError, match="null x, y or scales"):
        rx.rslx_rms_norm_e4m3(x, None, w, 1e-5, None, Z(4, 8).to(torch.float8_e4m3fn), None, None)
    with pytest.raises(rx.RslxError, match="y is"):
        rx.rslx_rms_norm_e4m3(x, None, w, 1e-5, None, Z(4, 8), Z(4), None)
    with pytest.raises(rx.RslxError, match="rows of y overlap"):
        rx.rslx_rms_norm(x, None, w, 1e-5, None, Z(1, 8).expand(4, 8), None)
    with pytest.raises(rx.RslxError, match="rows of total overlap"):
        rx.rslx_rms_norm(x, None, w, 1e-5, Z(1, 8).expand(4, 8), Z(4, 8), None)
    b = Z(200)
    m = lambda at: b[at:at + 32].view(4, 8)  # noqa: E731
    with pytest.raises(rx.RslxError, match="y and x overlap"):
        rx.rslx_rms_norm(m(0), None, w, 1e-5, None, m(4), None)
    with pytest.raises(rx.RslxError, match="total and residual overlap"):
        rx.rslx_rms_norm(x, m(0), w, 1e-5, m(8), Z(4, 8), None)
    with pytest.raises(rx.RslxError, match="y overlaps total"):
        rx.rslx_rms_norm(x, None, w, 1e-5, m(0), m(0), None)
    with pytest.raises(rx.RslxError, match="y overlaps weight"):
        rx.rslx_rms_norm(x, None, b[8:16], 1e-5, None, m(0), None)
    with pytest.raises(rx.RslxError, match="rstd overlaps x"):
        rx.rslx_rms_norm(m(0), None, w, 1e-5, None, Z(4, 8), b[8:12])
    with pytest.raises(rx.RslxError, match="y overlaps x"):
        rx.rslx_rms_norm_e4m3(m(0), None, w, 1e-5, None, b[:8].view(torch.float8_e4m3fn).view(4, 8), Z(4), None)
    with pytest.raises(rx.RslxError, match="16-byte"):
        rx.rslx_rms_norm(x, None, b[1:9], 1e-5, None, Z(4, 8), None)


def test_norm_backward_refusals():
    x, w, r, ws = Z(4, 8), Z(8), Z(4), Z(4096, dtype=torch.uint8)
    with pytest.raises(rx.RslxError, match="null dy"):
        rx.rslx_rms_norm_backward(None, x, w, r, None, Z(4, 8), Z(8), ws)
    with pytest.raises(rx.RslxError, match="null dy, total or rstd"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, None, None, Z(4, 8), Z(8), ws)
    with pytest.raises(rx.RslxError, match="dtotal is"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, r, Z(4, 8, dtype=F16), Z(4, 8), Z(8), ws)
    with pytest.raises(rx.RslxError, match="workspace"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, r, None, Z(4, 8), Z(8), None)
    with pytest.raises(rx.RslxError, match="workspace"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, r, None, Z(4, 8), Z(8), ws[:16])
    with pytest.raises(rx.RslxError, match="rows of dx overlap"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, r, None, Z(1, 8).expand(4, 8), None, None)
    b = Z(100)
    m = lambda at: b[at:at + 32].view(4, 8)  # noqa: E731
    with pytest.raises(rx.RslxError, match="dx and dtotal overlap"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, r, m(0), m(4), None, None)
    with pytest.raises(rx.RslxError, match="dweight overlaps dy"):
        rx.rslx_rms_norm_backward(m(0), x, w, r, None, None, b[8:16], ws)
    with pytest.raises(rx.RslxError, match="dx overlaps rstd"):
        rx.rslx_rms_norm_backward(Z(4, 8), x, w, b[4:8], None, m(0), None, None)
    for rows, cols in ((-1, 8), (4, 0), (4, 16385)):
        with pytest.raises(rx.RslxError):
            rx.rslx_rms_norm_backward_workspace_bytes(rows, cols)


# ---- Muon step ----------------------------------------------------------------------------------------------------------
def _muon(mats, ws=None, **kw):
    mu = rx.Muon(mats, kw.pop("lr", 0.1), **kw)
    rx.rslx_muon_step(mu, Z(rx.rslx_muon_step_workspace_bytes(mu), dtype=torch.uint8) if ws is None else ws)


def test_muon_refusals():
    w, g, m = Z(4, 6), Z(4, 6), Z(4, 6)
    ok = (w, w, g, m, m, 1.0)
    with pytest.raises(rx.RslxError, match="not a matrix"):
        rx.Muon([(None, w, Z(24), None, None, 1.0)], 0.1)
    with pytest.raises(rx.RslxError, match="m_in of matrix 1"):
        rx.Muon([ok, (w, w, g, Z(6, 4), m, 1.0)], 0.1)
    with pytest.raises(rx.RslxError, match="w_out of matrix 0"):
        rx.Muon([(w, w.to(BF16), g, m, m, 1.0)], 0.1)
    with pytest.raises(rx.RslxError, match="null w_out or grad"):
        _muon([(w, None, g, m, m, 1.0)])
    with pytest.raises(rx.RslxError, match="33 matrices"):
        _muon([ok] * 33)
    for steps in (0, -1, 33):
        with pytest.raises(rx.RslxError, match="%d steps" % steps):
            _muon([ok], steps=steps)
    with pytest.raises(rx.RslxError, match="0 x 6"):
        _muon([(None, Z(0, 6), Z(0, 6), None, None, 1.0)])
    mu = rx.Muon([ok], 0.1)
    mu.c[0].cols = 65537
    with pytest.raises(rx.RslxError, match="4 x 65537"):
        rx.rslx_muon_step_workspace_bytes(mu)
    mu = rx.Muon([ok], 0.1)
    mu.c[0].grad += 2
    with pytest.raises(rx.RslxError, match="grad not aligned"):
        rx.rslx_muon_step(mu, Z(1 << 16, dtype=torch.uint8))
    mu = rx.Muon([ok], 0.1)
    n = rx.rslx_muon_step_workspace_bytes(mu)
    for ws, text in ((None, "workspace"), (Z(n - 1, dtype=torch.uint8), "workspace"), (Z(n + 8, dtype=torch.uint8)[8:], "not 16-byte")):
        with pytest.raises(rx.RslxError, match=text):
            rx.rslx_muon_step(mu, ws)
    assert rx.lib.rslx_muon_step(None, 1, mu.cfg, None, 0, None) == 1
    assert rx.lib.rslx_muon_step(mu.c, 1, None, None, 0, None) == 1
    assert rx.lib.rslx_muon_step(None, 0, mu.cfg, None, 0, None) == 0
    assert rx.lib.rslx_muon_step(mu.c, -1, mu.cfg, None, 0, None) == 2


def test_muon_overlaps():
    b = Z(200)
    v = lambda at: b[at:at + 24].view(4, 6)  # noqa: E731
    g = lambda: Z(4, 6)  # noqa: E731
    refused = [
        [(v(0), v(4), g(), None, None, 1.0)],                                  # w_out beside w_in
        [(None, v(0), v(20), None, None, 1.0)],                                # w_out and grad
        [(g(), g(), v(0), v(0), v(0), 1.0)],                                   # m_out and grad
        [(None, v(0), g(), None, v(10), 1.0)],                                 # two outputs
        [(v(0), v(0), g(), None, None, 1.0), (v(23), v(23), g(), None, None, 1.0)],     # of two matrices
        [(g(), g(), g(), v(0), v(0), 1.0), (v(0), g(), g(), None, None, 1.0)],          # an input of the other
        [(v(0), v(0), g(), None, None, 1.0)] * 2,                              # the same matrix twice
    ]
    for mats in refused:
        with pytest.raises(rx.RslxError, match="overlaps"):
            _muon(mats)
    # side by side, in place and with shared inputs they are taken (and end at the launch, without a GPU)
    taken = [(v(0), v(0), v(72), v(24), v(24), 1.0), (v(48), v(48), v(72), None, None, 1.0), (v(72), v(96), v(72), v(72), v(120), 1.0)]
    with pytest.raises(rx.RslxError, match="status 4"):
        _muon(taken)


def test_muon_workspace_grows_with_the_matrices():
    def n(*shapes):
        mu = rx.Muon([], 0.1)
        mu.matrices, mu.c = [None] * len(shapes), (B._CMuonMatrix * len(shapes))()
        for i, (rows, cols) in enumerate(shapes):
            mu.c[i].rows, mu.c[i].cols = rows, cols
        return rx.rslx_muon_step_workspace_bytes(mu)
    assert 256 <= n((1, 1)) < n((64, 64)) < n((64, 64), (64, 64)) < n((4096, 4096))
    assert n((65536, 65536)) > 1 << 34                         # sizes beyond 32 bits
