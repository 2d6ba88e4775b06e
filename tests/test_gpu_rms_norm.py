"""Root-mean-square norm with the residual's addition on the GPU against fp64.

Bounds: the sum of a row's squares passes at most 60 roundings of u = 2^-24 (a lane's 32 values in order, a tree over lanes and wavefronts), its terms two
more and the addition of the residual two; half of that reaches 1 / sqrt, whose division and root add two: 35 u of rstd.
"""
import numpy as np
import pytest
import torch

from oracle import rms_norm as orn
from sequence_util import TYPES, U, check, f64, rounding, typed

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 2), (5, 7), (64, 128), (64, 256), (17, 48), (70, 235), (9, 255), (2, 512), (40, 1000), (300, 24), (11, 2048), (6, 4096), (4, 4098),
         (3, 8192), (2, 9001), (2, 16384), (2600, 130), (4500, 40)]
EPS = float(np.float32(1e-5))
R = 36 * U


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


def _case(seed, rows, cols, dtype):
    g = np.random.default_rng(seed)
    r = lambda: typed(g.normal(size=(rows, cols)) * g.uniform(0.3, 3, (rows, 1)), TYPES[dtype])  # noqa: E731
    return r(), r(), r(), r(), typed(1 + 0.3 * g.normal(size=cols), torch.float32)


def _forward_check(x, residual, weight, got):
    y, z, r = orn.forward(f64(x), f64(residual), f64(weight), EPS)
    if got[0] is not None:
        check("y", got[0], y, rounding(x.dtype, y) + (R + 4 * U) * np.abs(y))
    if got[1] is not None:
        check("total", got[1], z, rounding(x.dtype, z) + U * np.abs(z))
    if got[2] is not None:
        check("rstd", got[2], r, R * r)


def _backward_check(dy, total, weight, rstd, dtotal, dx, dweight):
    dy, total, rstd = f64(dy), f64(total), f64(rstd)
    ref, dw = orn.backward(dy, total, f64(weight), rstd, f64(dtotal))
    h = np.abs(total) * rstd[:, None]
    k = np.abs(dy) * (1 if weight is None else np.abs(f64(weight)))
    if dx is not None:
        b = rstd[:, None] * U * (6 * k + h * 72 * (k * h).mean(1, keepdims=True)) + 2 * U * (np.abs(ref) + (0 if dtotal is None else np.abs(f64(dtotal))))
        check("dx", dx, ref, rounding(dx.dtype, ref) + b)
    if dweight is not None:
        # a lane adds the rows that its workgroup takes, at most 18 here, then at most 16 sets of lanes, 16 workgroups' sums a lane and 64 lanes in two
        # steps of eight, and the products' own
        check("dweight", dweight, dw, 100 * U * (np.abs(dy) * h).sum(0))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(rx, rows, cols, dtype):
    x, res, dy, dt, w = _case(rows * 1000 + cols, rows, cols, dtype)
    gx, gr, gd, gt, gw = (t.cuda() for t in (x, res, dy, dt, w))
    nan = lambda *s, like=x.dtype: torch.full(s, float("nan"), dtype=like, device="cuda")  # noqa: E731
    for residual in (res, None):
        y, total, rstd = nan(rows, cols), nan(rows, cols), nan(rows, like=torch.float32)
        rx.rslx_rms_norm(gx, None if residual is None else gr, gw, EPS, total, y, rstd)
        _forward_check(x, residual, w, (y, total, rstd))
        dx, dw = nan(rows, cols), nan(cols, like=torch.float32)
        ws = rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(rows, cols))
        rx.rslx_rms_norm_backward(gd, total, gw, rstd, None if residual is None else gt, dx, dw, ws)
        _backward_check(dy, total, w, rstd, None if residual is None else dt, dx, dw)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_bytes(rx, rows, cols, dtype):
    x, res, _, _, w = _case(rows * 1000 + cols + 1, rows, cols, dtype)
    y = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
    total, rstd, scales = torch.empty_like(x, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    rx.rslx_rms_norm_e4m3(x.cuda(), res.cuda(), w.cuda(), EPS, total, y, scales, rstd)
    _forward_check(x, res, w, (None, total, rstd))
    ref = orn.forward(f64(x), f64(res), f64(w), EPS)[0]
    scale = np.abs(ref).max(1) / 448
    check("scales", scales, scale, (R + 6 * U) * scale)
    # half a step of a value: 2^-4 of it, or half of the smallest number, 2^-10 scales
    check("y", y.float() * scales[:, None], ref, 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * scale[:, None] + 60 * U * np.abs(ref))
    # and each is the nearest that the type has
    near = (f64(y) == f64(torch.as_tensor(ref / scale[:, None]).float().to(torch.float8_e4m3fn).float())).mean()
    assert near > 1 - 1e-3 - 2 / (rows * cols)


def test_a_byte_is_the_nearest(rx):
    """Weights that put known quotients into a row: every positive e4m3 number, the borders between two, and next to them."""
    steps = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    mid = (steps[1:] + steps[:-1]) / 2
    values = torch.cat([steps, mid, mid * (1 + 2 ** -12), mid * (1 - 2 ** -12), -steps, -mid])
    w = values.float()
    x = torch.ones(2, len(w))
    y = torch.empty(2, len(w), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(2, device="cuda")
    rx.rslx_rms_norm_e4m3(x.cuda(), None, w.cuda(), 0.0, None, y, scales, None)
    # r = 1 / sqrt(1), so the largest is 448 and the scale 1
    assert torch.equal(scales, torch.ones_like(scales))
    assert torch.equal(y[0].float().cpu(), w.to(torch.float8_e4m3fn).float()) and torch.equal(y[0].float(), y[1].float())


def test_rows_of_zeros_and_rows_that_are_not_finite(rx):
    x, res, dy, _, w = _case(9, 6, 300, "fp32")
    x[1], res[1] = 0, 0
    x[2, 7], x[3, 8] = float("nan"), float("inf")
    x[4], res[4] = 1e-38, 0
    y8, y = torch.empty(6, 300, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, 300, device="cuda")
    scales, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    rx.rslx_rms_norm_e4m3(x.cuda(), res.cuda(), w.cuda(), 0.0, None, y8, scales, rstd)
    rx.rslx_rms_norm(x.cuda(), res.cuda(), w.cuda(), EPS, None, y, rstd)
    ok = [0, 5]
    ref = orn.forward(f64(x)[ok], f64(res)[ok], f64(w), EPS)[0]
    check("y", y[ok], ref, (R + 4 * U) * np.abs(ref))
    assert not y[1].any() and torch.isnan(y[2]).all() and torch.isnan(y[3, 8]) and not y[3, :8].any()
    assert torch.isnan(scales[2]) and torch.isnan(y8[2].float()).all()
    rx.rslx_rms_norm_e4m3(x.cuda(), res.cuda(), w.cuda(), EPS, None, y8, scales, rstd)
    assert not y8[1].float().any() and scales[1] == 2.0 ** -126
    assert torch.isfinite(scales[4]) and torch.isfinite(y8[4].float()).all()
    assert torch.isnan(scales[3]) or torch.isinf(scales[3])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [64, 100, 512])
def test_rows_apart_and_unaligned(rx, dtype, cols):
    rows = 21
    x, res, dy, dt, w = _case(cols, rows, cols, dtype)
    for pad, shift in ((8, 0), (3, 0), (1, 1)):
        def place(t, fill=float("nan")):
            wide = torch.full((rows, cols + pad), fill, dtype=t.dtype, device="cuda")
            wide[:, shift:shift + cols] = t.cuda()
            return wide, wide[:, shift:shift + cols]
        (_, gx), (_, gr), (_, gd), (_, gt) = place(x), place(res), place(dy), place(dt)
        (wy, y), (wt, total), (wd, dx) = place(torch.zeros_like(x)), place(torch.zeros_like(x)), place(torch.zeros_like(x))
        rstd, scales, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        rx.rslx_rms_norm(gx, gr, w.cuda(), EPS, total, y, rstd)
        _forward_check(x, res, w, (y, total, rstd))
        rx.rslx_rms_norm_backward(gd, total, w.cuda(), rstd, gt, dx, dw, rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(rows, cols)))
        _backward_check(dy, total, w, rstd, dt, dx, dw)
        w8 = torch.full((rows, cols + pad), 1.0, device="cuda").to(torch.float8_e4m3fn)
        y8, dense = w8[:, shift:shift + cols], torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
        rx.rslx_rms_norm_e4m3(gx, gr, w.cuda(), EPS, None, y8, scales, None)
        rx.rslx_rms_norm_e4m3(x.cuda(), res.cuda(), w.cuda(), EPS, None, dense, scales, None)
        assert (y8.float() - dense.float()).abs().max() <= 32        # a tie at most: sums in another order
        for wide in (wy, wt, wd):                              # nothing between the rows is written
            assert torch.isnan(wide[:, :shift]).all() and torch.isnan(wide[:, shift + cols:]).all()
        assert (w8[:, :shift].float() == 1).all() and (w8[:, shift + cols:].float() == 1).all()


@pytest.mark.parametrize("rows,cols", [(50, 96), (3000, 512), (7, 3001)])
def test_parts_may_be_left_out_and_in_place(rx, rows, cols):
    x, res, dy, dt, w = _case(5, rows, cols, "fp32")
    gx, gr, gd, gt, gw = (t.cuda() for t in (x, res, dy, dt, w))
    y, total, rstd = torch.empty_like(gx), torch.empty_like(gx), torch.empty(rows, device="cuda")
    rx.rslx_rms_norm(gx, gr, gw, EPS, total, y, rstd)
    out = torch.empty_like(gx)
    rx.rslx_rms_norm(gx, gr, None, EPS, None, out, None)
    _forward_check(x, res, None, (out, None, None))
    for a, b in ((0, 1), (1, 0), (0, None), (1, None), (None, 0), (None, 1)):      # y and total in place of x or residual
        both = [gx.clone(), gr.clone()]
        oy, ot = both[a] if a is not None else torch.empty_like(gx), both[b] if b is not None else None
        rx.rslx_rms_norm(both[0], both[1], gw, EPS, ot, oy, None)
        assert torch.equal(oy, y) and (ot is None or torch.equal(ot, total))
    ws = rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(rows, cols))
    dx, dw = torch.empty_like(gx), torch.empty(cols, device="cuda")
    rx.rslx_rms_norm_backward(gd, total, gw, rstd, gt, dx, dw, ws)
    for k in range(3):
        ins = [gd.clone(), total.clone(), gt.clone()]
        dw2 = torch.empty(cols, device="cuda")
        rx.rslx_rms_norm_backward(ins[0], ins[1], gw, rstd, ins[2], ins[k], dw2, ws)
        assert torch.equal(ins[k], dx) and torch.equal(dw, dw2)
    only = torch.empty_like(gx)
    rx.rslx_rms_norm_backward(gd, total, gw, rstd, gt, only, None, None)
    assert torch.equal(only, dx)
    dw2 = torch.empty(cols, device="cuda")
    rx.rslx_rms_norm_backward(gd, total, gw, rstd, gt, None, dw2, ws)
    assert torch.equal(dw, dw2)
    rx.rslx_rms_norm_backward(gd, total, None, rstd, None, only, dw2, ws)
    _backward_check(dy, total, None, rstd, None, only, dw2)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(37, 3), (300, 9), (5000, 61), (900, 235), (400, 511), (90, 1003), (33, 4093), (5, 16383)])
def test_rows_that_start_anywhere_in_place(rx, rows, cols, dtype):
    """The last piece of such a row begins inside the one before it: what a neighbour stores there meanwhile is of no account."""
    x, res, dy, dt, w = _case(cols, rows, cols, dtype)
    gx, gr, gd, gt, gw = (t.cuda() for t in (x, res, dy, dt, w))
    y, total, rstd = torch.empty_like(gx), torch.empty_like(gx), torch.empty(rows, device="cuda")
    rx.rslx_rms_norm(gx, gr, gw, EPS, total, y, rstd)
    _forward_check(x, res, w, (y, total, rstd))
    for a, b in ((0, 1), (1, 0)):
        both = [gx.clone(), gr.clone()]
        rx.rslx_rms_norm(both[0], both[1], gw, EPS, both[b], both[a], None)
        assert torch.equal(both[a], y) and torch.equal(both[b], total)
    ws = rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(rows, cols))
    dx, dw, dw2 = torch.empty_like(gx), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    rx.rslx_rms_norm_backward(gd, total, gw, rstd, gt, dx, dw, ws)
    _backward_check(dy, total, w, rstd, dt, dx, dw)
    for k in range(3):
        ins = [gd.clone(), total.clone(), gt.clone()]
        rx.rslx_rms_norm_backward(ins[0], ins[1], gw, rstd, ins[2], ins[k], dw2, ws)
        assert torch.equal(ins[k], dx) and torch.equal(dw, dw2)


def test_no_rows(rx):
    e = torch.empty(0, 40, device="cuda")
    rx.rslx_rms_norm(e, e, None, EPS, None, e, None)
    dw = torch.full((40,), 7.0, device="cuda")
    rx.rslx_rms_norm_backward(e, e, None, torch.empty(0, device="cuda"), None, e, dw, rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(0, 40)))
    assert not dw.any()


def test_graph_replays(rx):
    x, res, dy, dt, w = (t.cuda() for t in _case(4, 400, 300, "bf16"))
    y, total, dx, rstd, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(400, device="cuda"), torch.empty(300, device="cuda")
    ws = rx.workspace(rx.rslx_rms_norm_backward_workspace_bytes(400, 300))

    def both():
        rx.rslx_rms_norm(x, res, w, EPS, total, y, rstd)
        rx.rslx_rms_norm_backward(dy, total, w, rstd, dt, dx, dw, ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        for t in (x, res, dy, dt):
            t.copy_(t.flip(0) * 0.5 + 0.25)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, total, dx, rstd, dw)]
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, total, dx, rstd, dw)))
