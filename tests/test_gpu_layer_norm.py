"""Layer norm on the GPU against fp64.

Bounds: a lane adds at most 32 values in order, lanes and wavefronts another 26 in a tree: 60 roundings of u = 2^-24 for a row's sum.
"""
import numpy as np
import pytest
import torch

from oracle import layer_norm as oln
from sequence_util import TYPES, U, check, f64, rounding, typed

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 2), (5, 7), (64, 128), (17, 48), (33, 64), (70, 235), (9, 256), (2, 512), (40, 1000), (300, 24), (11, 2048), (6, 4096), (4, 4098),
         (3, 8192), (2, 9001), (2, 16384)]


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


def _case(seed, rows, cols, dtype, far=3.0):
    g = np.random.default_rng(seed)
    x = typed(g.normal(size=(rows, cols)) * g.uniform(0.5, 2, (rows, 1)) + far * g.normal(size=(rows, 1)), TYPES[dtype])
    dy = typed(g.normal(size=(rows, cols)), TYPES[dtype])
    w, b = typed(1 + 0.3 * g.normal(size=cols), torch.float32), typed(g.normal(size=cols), torch.float32)
    return x, dy, w, b


def _forward_bounds(x, w, b, eps, dtype):
    x = f64(x)
    y, m, r = oln.forward(x, w, b, eps)
    size = np.abs(x).mean(1, keepdims=True)
    w = np.ones(x.shape[1]) if w is None else np.abs(w)
    b = np.zeros(x.shape[1]) if b is None else np.abs(b)
    h = np.abs(x - m[:, None]) * r[:, None]
    dm = 62 * U * size                                         # of the mean
    dr = 50 * U + (dm[:, 0] * r) ** 2                          # relative, of rstd: half of the variance's 60 + 4 roundings and the mean's square, sqrt and division
    by = rounding(dtype, y) + w * (r[:, None] * dm + h * (dr[:, None] + 4 * U)) + 2 * U * (h * w + b)
    return (y, m, r), (by, dm[:, 0], dr * r)


def _backward_bounds(dy, x, w, m, r, dtype):
    dy, x, m, r = f64(dy), f64(x), f64(m), f64(r)
    dx, dw, db = oln.backward(dy, x, w, m, r)
    h = np.abs(x - m[:, None]) * r[:, None]
    g = np.abs(dy) * (1 if w is None else np.abs(w))
    mean = lambda v: v.mean(1, keepdims=True)  # noqa: E731
    bx = rounding(dtype, dx) + r[:, None] * U * (6 * g + 66 * mean(g) + h * 72 * mean(g * h))
    # a lane adds the rows that its workgroup takes, at most 16 for up to 8192 rows, then at most 16 sets of lanes, then 32 workgroups'
    # sums a lane and 16 lanes: 80, and the products' own
    return (dx, dw, db), (bx, 100 * U * (np.abs(dy) * h).sum(0), 100 * U * np.abs(dy).sum(0))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(rx, rows, cols, dtype):
    x, dy, w, b = _case(rows * 1000 + cols, rows, cols, dtype)
    eps = float(np.float32(1e-5))
    y, mean, rstd = torch.empty_like(x, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gx, gd, gw, gb = x.cuda(), dy.cuda(), w.cuda(), b.cuda()
    rx.rslx_layer_norm(gx, gw, gb, eps, y, mean, rstd)
    ref, bound = _forward_bounds(x, f64(w), f64(b), eps, x.dtype)
    for name, got, r, t in zip(("y", "mean", "rstd"), (y, mean, rstd), ref, bound):
        check(name, got, r, t)
    dx, dw, db = torch.empty_like(y), torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ws = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(rows, cols))
    rx.rslx_layer_norm_backward(gd, gx, gw, mean, rstd, dx, dw, db, ws)
    ref, bound = _backward_bounds(dy, x, f64(w), mean, rstd, x.dtype)
    for name, got, r, t in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, bound):
        check(name, got, r, t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [64, 100, 512])
def test_rows_apart_and_unaligned(rx, dtype, cols):
    x, dy, w, b = _case(cols, 21, cols, dtype)
    for pad, shift in ((8, 0), (3, 0), (1, 1)):
        def place(t):
            wide = torch.full((21, cols + pad), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, shift:shift + cols] = t.cuda()
            return wide, wide[:, shift:shift + cols]
        (_, gx), (_, gd), (ywide, y), (dxwide, dx) = place(x), place(dy), place(torch.zeros_like(x)), place(torch.zeros_like(x))
        mean, rstd = torch.empty(21, device="cuda"), torch.empty(21, device="cuda")
        rx.rslx_layer_norm(gx, w.cuda(), b.cuda(), 1e-5, y, mean, rstd)
        ref, bound = _forward_bounds(x, f64(w), f64(b), float(np.float32(1e-5)), x.dtype)
        check("y", y, ref[0], bound[0])
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        rx.rslx_layer_norm_backward(gd, gx, w.cuda(), mean, rstd, dx, dw, db, rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(21, cols)))
        ref, bound = _backward_bounds(dy, x, f64(w), mean, rstd, x.dtype)
        for name, got, r, t in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, bound):
            check(name, got, r, t)
        for wide in (ywide, dxwide):                           # nothing between the rows is written
            assert torch.isnan(wide[:, :shift]).all() and torch.isnan(wide[:, shift + cols:]).all()


def test_parts_may_be_left_out(rx):
    x, dy, w, b = _case(5, 50, 96, "fp32")
    eps = float(np.float32(1e-5))
    gx, gd = x.cuda(), dy.cuda()
    y, mean, rstd = torch.empty_like(gx), torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    for weight, bias in ((None, None), (w, None), (None, b)):
        rx.rslx_layer_norm(gx, None if weight is None else weight.cuda(), None if bias is None else bias.cuda(), eps, y, mean, rstd)
        ref, bound = _forward_bounds(x, f64(weight), f64(bias), eps, x.dtype)
        check("y", y, ref[0], bound[0])
        rx.rslx_layer_norm(gx, None if weight is None else weight.cuda(), None if bias is None else bias.cuda(), eps, y, None, None)
        check("y", y, ref[0], bound[0])
    ws = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(50, 96))
    ref, bound = _backward_bounds(dy, x, None, mean, rstd, x.dtype)
    for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0)):
        out = [torch.empty(s, device="cuda") if a else None for a, s in zip(asked, ((50, 96), 96, 96))]
        rx.rslx_layer_norm_backward(gd, gx, None, mean, rstd, *out, ws if asked[1] or asked[2] else None)
        for name, got, r, t in zip(("dx", "dweight", "dbias"), out, ref, bound):
            if got is not None:
                check(name, got, r, t)


def test_in_place(rx):
    x, dy, w, b = _case(6, 130, 300, "bf16")
    gx, gd, gw, gb = x.cuda(), dy.cuda(), w.cuda(), b.cuda()
    y, mean, rstd = torch.empty_like(gx), torch.empty(130, device="cuda"), torch.empty(130, device="cuda")
    rx.rslx_layer_norm(gx, gw, gb, 1e-5, y, mean, rstd)
    z = gx.clone()
    rx.rslx_layer_norm(z, gw, gb, 1e-5, z, None, None)
    assert torch.equal(y, z)
    ws = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(130, 300))
    dx, dw, db = torch.empty_like(gx), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    rx.rslx_layer_norm_backward(gd, gx, gw, mean, rstd, dx, dw, db, ws)
    for over in (gd.clone(), gx.clone()):
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        d, xx = (over, gx) if torch.equal(over, gd) else (gd, over)
        rx.rslx_layer_norm_backward(d, xx, gw, mean, rstd, over, dw2, db2, ws)
        assert torch.equal(over, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_rows_far_from_zero_and_constant_rows(rx):
    rows, cols = 8, 96
    g = np.random.default_rng(8)
    x = typed(1000 + 1e-2 * g.normal(size=(rows, cols)), torch.float32)
    x[3] = 5.0
    y, mean, rstd = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    eps = float(np.float32(1e-5))
    rx.rslx_layer_norm(x.cuda(), None, None, eps, y, mean, rstd)
    ref, bound = _forward_bounds(x, None, None, eps, x.dtype)
    for name, got, r, t in zip(("y", "mean", "rstd"), (y, mean, rstd), ref, bound):
        check(name, got, r, t)
    assert torch.equal(y[3].cpu(), torch.zeros(cols))


def test_what_is_not_finite_stays_in_its_row(rx):
    x, dy, w, b = _case(9, 67, 40, "fp32")
    x[5, 3], x[66, 0] = float("nan"), float("inf")
    y, mean, rstd = torch.empty(67, 40, device="cuda"), torch.empty(67, device="cuda"), torch.empty(67, device="cuda")
    rx.rslx_layer_norm(x.cuda(), w.cuda(), b.cuda(), 1e-5, y, mean, rstd)
    bad = ~torch.isfinite(y).all(1).cpu()
    assert bad.nonzero().flatten().tolist() == [5, 66]


def test_no_rows(rx):
    dw, db = torch.full((12,), 7.0, device="cuda"), torch.full((12,), 7.0, device="cuda")
    e, r = torch.empty(0, 12, device="cuda"), torch.empty(0, device="cuda")
    rx.rslx_layer_norm_backward(e, e, None, r, r, None, dw, db, rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(0, 12)))
    assert not dw.any() and not db.any()


def test_many_rows_same_bits_and_a_graph(rx):
    x, dy, w, b = _case(10, 20011, 64, "bf16")
    gx, gd, gw, gb = x.cuda(), dy.cuda(), w.cuda(), b.cuda()
    y, mean, rstd, dx = torch.empty_like(gx), torch.empty(20011, device="cuda"), torch.empty(20011, device="cuda"), torch.empty_like(gx)
    dw, db = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ws = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(20011, 64))

    def both():
        rx.rslx_layer_norm(gx, gw, gb, 1e-5, y, mean, rstd)
        rx.rslx_layer_norm_backward(gd, gx, gw, mean, rstd, dx, dw, db, ws)

    both()
    ref, bound = _backward_bounds(dy, x, f64(w), mean, rstd, x.dtype)
    # 20 011 rows over 512 workgroups: at most 40 rows in order, 24 more than the bound counts
    for name, got, r, t in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, bound):
        check(name, got, r, t if name == "dx" else 1.24 * t)
    want = [t.clone() for t in (y, mean, rstd, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip((y, mean, rstd, dx, dw, db), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (y, mean, rstd, dx, dw, db):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((y, mean, rstd, dx, dw, db), want))
        both()
        torch.cuda.synchronize()


def test_rows_further_apart_than_32_bits_reach(rx):
    far = (1 << 31) + 40
    big = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    x, dy, w, b = _case(11, 3, 40, "bf16")
    gx, gy = torch.as_strided(big, (3, 40), (far, 1), 0), torch.as_strided(big, (3, 40), (far, 1), 64)
    gx.copy_(x)
    rx.rslx_layer_norm(gx, w.cuda(), b.cuda(), 1e-5, gy, None, None)
    ref, bound = _forward_bounds(x, f64(w), f64(b), float(np.float32(1e-5)), x.dtype)
    check("y", gy, ref[0], bound[0])
