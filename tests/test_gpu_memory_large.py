"""Large calls of the operators around a gated memory: outputs and inputs that go past the caches, rows too far apart for 32-bit offsets, every tile of the Muon
step's products."""
import numpy as np
import pytest
import torch

from oracle import gated_recurrence as ogr, muon as om, rms_norm as orn
from sequence_util import U, check, f64, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


def _recurrence(rx, xg, dh, s0, dones):
    """Both directions of sequences [T, N, 2 D] whose candidates and gates lie side by side."""
    T, N, D = dh.shape
    gr = rx.GatedRec(dh.dtype, T, N, D, dones)
    x, g = xg[..., :D], xg[..., D:]
    h, dx, dg = torch.empty_like(dh), torch.empty_like(dh), torch.empty_like(dh)
    s, ds0 = torch.empty_like(s0), torch.empty_like(s0)
    rx.rslx_gated_recurrence(gr, x, g, s0, h, s, rx.workspace(rx.rslx_gated_recurrence_workspace_bytes(gr)))
    rx.rslx_gated_recurrence_backward(gr, x, g, s0, dh, s0, dx, dg, ds0, rx.workspace(rx.rslx_gated_recurrence_backward_workspace_bytes(gr)))
    return h, s, dx, dg, ds0


@pytest.mark.parametrize("T,N,D,dtype", [(24, 4096, 256, torch.float32), (20, 16384, 256, torch.bfloat16)])
def test_a_large_roll_out_is_its_environments(rx, T, N, D, dtype):
    """Environments do not see each other: a call that passes the caches gives the bits of calls that do not."""
    g = torch.Generator("cuda").manual_seed(1)
    xg, dh = torch.randn(T, N, 2 * D, generator=g, device="cuda").to(dtype), torch.randn(T, N, D, generator=g, device="cuda").to(dtype)
    s0 = torch.randn(N, D, generator=g, device="cuda")
    dones = (torch.rand(T, N, generator=g, device="cuda") < 0.02).to(torch.uint8)
    whole = _recurrence(rx, xg, dh, s0, dones)
    step = N // 16
    for n in range(0, N, 3 * step):
        part = slice(n, n + step)
        few = _recurrence(rx, xg[:, part].contiguous(), dh[:, part].contiguous(), s0[part].contiguous(), dones[:, part].contiguous())
        for a, b, time_first in zip(whole, few, (1, 0, 1, 1, 0)):
            assert torch.equal(a[:, part] if time_first else a[part], b)


def test_a_large_norm_is_its_rows(rx):
    g = torch.Generator("cuda").manual_seed(2)
    rows, cols = 70000, 520
    x, r, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")

    def run(x, r, dy):
        y, total, dx, y8 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
        rstd, scales = torch.empty(x.shape[0], device="cuda"), torch.empty(x.shape[0], device="cuda")
        rx.rslx_rms_norm(x, r, w, 1e-5, total, y, rstd)
        rx.rslx_rms_norm_e4m3(x, r, w, 1e-5, None, y8, scales, None)
        rx.rslx_rms_norm_backward(dy, total, w, rstd, r, dx, None, None)
        return y, total, dx, y8.view(torch.uint8), rstd, scales
    whole = run(x, r, dy)
    for a in range(0, rows, 23000):
        for p, q in zip(whole, run(x[a:a + 500], r[a:a + 500], dy[a:a + 500])):
            assert torch.equal(p[a:a + 500], q)


def _far(rows, cols, dtype, apart):
    """rows whose distance needs more than 32 bits in bytes."""
    wide = torch.empty((rows - 1) * apart + cols, dtype=dtype, device="cuda")
    return wide.as_strided((rows, cols), (apart, 1))


@pytest.mark.parametrize("apart", [(1 << 31) + 8, (1 << 31) + 7])
def test_rows_far_apart(rx, apart):
    T, N, D, dt = 3, 2, 40, torch.bfloat16
    gen = np.random.default_rng(3)
    place = lambda v: _far(T, N * D, dt, apart).copy_(torch.as_tensor(v.reshape(T, N * D))).unflatten(1, (N, D))  # noqa: E731
    val = lambda: torch.as_tensor(gen.normal(size=(T, N, D))).to(dt).double().numpy()  # noqa: E731
    x, g, dh, s0 = val(), val(), val(), gen.normal(size=(N, D)).astype(np.float32)
    gx, gg, gd = place(x), place(g), place(dh)
    h, dx, dg = place(x), place(x), place(x)
    gr = rx.GatedRec(dt, T, N, D)
    gs, s, ds0 = torch.as_tensor(s0).cuda(), torch.empty(N, D, device="cuda"), torch.empty(N, D, device="cuda")
    ws = rx.workspace(max(rx.rslx_gated_recurrence_workspace_bytes(gr), rx.rslx_gated_recurrence_backward_workspace_bytes(gr)))
    rx.rslx_gated_recurrence(gr, gx, gg, gs, h, s, ws)
    rx.rslx_gated_recurrence_backward(gr, gx, gg, gs, gd, None, dx, dg, ds0, ws)
    ref, last, _ = ogr.forward(x, g, s0)
    m, e, e_last = ogr.sizes(x, g, s0, each=24 * U)
    check("h", h, ref, rounding(dt, ref) + e)
    check("s", s, last, e_last)
    for name, got, r in zip(("dx", "dg", "ds0"), (dx, dg, ds0), ogr.backward(x, g, dh, None, s0)):
        # three steps of 24 u each, of values below 40
        check(name, got, r, rounding(dt, r) + 3 * 48 * U * 40)
    del h, dx, dg
    rows, total, y, dz = gx.flatten(1), gg.flatten(1), gd.flatten(1), place(x).flatten(1)
    rstd, dw = torch.empty(T, device="cuda"), torch.empty(N * D, device="cuda")
    res = torch.as_tensor(g.reshape(T, -1)).to(dt).cuda()
    rx.rslx_rms_norm(rows, res, None, 1e-5, total, y, rstd)
    ry, rz, rr = orn.forward(x.reshape(T, -1), g.reshape(T, -1), None, float(np.float32(1e-5)))
    check("y", y, ry, rounding(dt, ry) + 40 * U * np.abs(ry))
    check("total", total, rz, rounding(dt, rz) + U * np.abs(rz))
    rx.rslx_rms_norm_backward(rows, total, None, rstd, res, dz, dw, rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(T, N * D)))
    rd, rw = orn.backward(x.reshape(T, -1), f64(total), None, f64(rstd), g.reshape(T, -1))
    check("dx", dz, rd, rounding(dt, rd) + 200 * U * (1 + np.abs(rd)))
    check("dweight", dw, rw, 100 * U * 40)


def _muon(rx, shapes, seed):
    """The updates of matrices of these shapes in one call, and whether each is within its bound of fp64's (on the GPU)."""
    g = torch.Generator("cuda").manual_seed(seed)
    us = [torch.randn(s, generator=g, device="cuda") for s in shapes]
    outs = [torch.full_like(u, float("nan")) for u in us]
    mu = rx.Muon([(None, o, u, None, None, 1.0) for u, o in zip(us, outs)], -1.0, nesterov=False, steps=5)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    for i, (u, o) in enumerate(zip(us, outs)):
        x = u.double() / u.double().norm()
        x = x.t().contiguous() if x.shape[0] > x.shape[1] else x
        bound = 0.0
        for _ in range(5):
            # as in test_gpu_muon.py, with the polynomial's slope at zero, its steepest
            bound = bound * om.A + 25 * 16 * U * x.norm().item()
            a = x @ x.t().contiguous()
            x = om.A * x + (om.B * a + om.C * (a @ a)) @ x
        got = o.double().t() if o.shape[0] > o.shape[1] else o.double()
        off = (got - x).norm().item()
        assert off <= bound and bound < 0.05 * x.norm().item(), (i, u.shape, off, bound)
        worst = (got - x).abs().max().item()
        assert worst <= bound, (i, u.shape, worst)


@pytest.mark.parametrize("shapes", [
    [(200, 190)] * 32,                                         # tiles of 64 x 64, cut off at both edges
    [(1500, 1490)],                                            # the same for both kinds of products
    [(500, 520)] * 31 + [(40, 33)],                            # tiles of 256 x 128, cut off at both edges, and a matrix inside one tile
    [(2000, 4200)], [(4200, 2010)],
    [(96, 5000), (5000, 96), (1, 3000), (3000, 1)],
], ids=lambda s: "%dx%dx%d" % (len(s), *s[0]))
def test_muons_tiles(rx, shapes):
    _muon(rx, shapes, len(shapes))
